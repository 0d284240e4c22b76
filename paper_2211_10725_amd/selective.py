"""A sequence model of selective leaky blocks on spike trains: the selective scan with its
short convolution and layer norms.

    x0  = E spikes_t                                   one dense synapse per step
    per block:  v | z = W_in layer_norm(x)             dense
                u     = silu(short causal convolution of v)
                d | b | c = W_x u                      dense: raw steps, both vectors
                s     = selective scan of u with steps softplus(d + dt_bias), gated by z
                x     = x + scale norm(W_out s) w_post
    readout:    Leaky neurons on layer_norm(x), loss on their spike counts

A block's integrators leak as the neurons' membranes do, but by steps that the input
chooses; whole sequences train and run in parallel over channels (and over time, where
these are few), and single steps go on from the states alone.

``python -m paper_2211_10725_amd.selective`` trains one on synthetic spike trains and
continues a prompt step by step.
"""
from __future__ import annotations

import numpy as np

import paper_2211_10725_amd as snn
from paper_2211_10725_amd.sequence import SequenceNet, spike_trains


class SelectiveNet(SequenceNet):
    """Parameters, buffers and call sequence of the model above, with the calls of
    ``SequenceNet``.

    n_in inputs, a residual stream of n values, `width` channels of `states` integrators in
    each block, convolutions of `taps` taps, `blocks` blocks, n_out output neurons.  The
    decay rates are a = -exp(log_a)."""

    def __init__(self, n_in, n, width, states, blocks, n_out, T, B, taps=4, beta=0.5, slope=3.0,
                 eps=1e-5, seed=0, device="cuda"):
        import torch
        self.torch, self.device = torch, device
        self.T, self.B, self.n, self.n_in, self.n_out, self.eps = T, B, n, n_in, n_out, eps
        self.width, self.n_states, self.taps = width, states, taps
        self.beta, self.slope = beta, slope
        rng = np.random.default_rng(seed)

        def param(a):
            return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.float32).to(device)

        def uniform(rows, cols):
            return param(rng.uniform(-1, 1, (rows, cols)) / np.sqrt(cols))

        def full(size, v):
            return param(np.full(size, v))

        L = range(blocks)
        self.E = uniform(n, n_in)
        self.W = [uniform(2 * width, n) for _ in L]
        self.W_x = [uniform(width + 2 * states, width) for _ in L]
        self.W_out = [uniform(n, width) for _ in L]
        self.conv_w = [param(rng.uniform(-1, 1, (taps, width)) / np.sqrt(taps)) for _ in L]
        self.conv_b = [full(width, 0.0) for _ in L]
        # rates 1 .. states in every channel, steps between 0.001 and 0.1: memories of ten
        # to a thousand tokens
        self.log_a = [param(np.log(np.arange(1.0, states + 1))[:, None] + np.zeros((1, width)))
                      for _ in L]
        rest = [np.exp(rng.uniform(np.log(1e-3), np.log(0.1), width)) for _ in L]
        self.dt_bias = [param(r + np.log(-np.expm1(-r))) for r in rest]
        self.skip = [full(width, 1.0) for _ in L]
        self.ln_w = [full(n, 1.0) for _ in range(blocks + 1)]
        self.ln_b = [full(n, 0.0) for _ in range(blocks + 1)]
        self.w_post, self.scale = [full(n, 1.0) for _ in L], [full(n, 0.5) for _ in L]
        self.R = uniform(n_out, n)
        self.params, self.grads = [], []

        def add(name):
            value = getattr(self, name)
            own = value if isinstance(value, list) else [value]
            g = [torch.empty_like(p) for p in own]
            self.params += own
            self.grads += g
            setattr(self, "g_" + name, g if isinstance(value, list) else g[0])

        for name in ("E", "W", "W_x", "W_out", "conv_w", "conv_b", "log_a", "dt_bias", "skip", "ln_w",
                     "ln_b", "w_post", "scale", "R"):
            add(name)
        self.plans = {}

    # ---- buffers and descriptors of one shape -------------------------------
    def _new_plan(self, T, B, train):
        torch = self.torch
        p = type("Plan", (), {})()
        p.bufs, p.stays = [], train
        L, n, m, N = len(self.W), self.n, self.width, self.n_states

        def new(*shape, dtype=torch.float32):
            p.bufs.append(torch.empty(shape, dtype=dtype, device=self.device))
            return p.bufs[-1]

        def dense(n_in, n_out, in_dtype=snn.F32):
            return snn.layer_desc(dict(kind="dense", n_in=n_in, n_out=n_out, neuron="leaky",
                                       beta=self.beta), T, B, in_dtype=in_dtype, slope=self.slope)

        p.embed, p.readout = dense(self.n_in, n, snn.U8), dense(n, self.n_out)
        p.w_in, p.w_x, p.w_out = dense(n, 2 * m), dense(m, m + 2 * N), dense(m, n)
        kept = L if train else 1
        p.x = [new(T, B, n) for _ in range(L + 1 if train else 2)]
        p.h = [new(T, B, n) for _ in range(L + 1 if train else 2)]
        p.vz, p.dbc = [new(T, B, 2 * m) for _ in range(kept)], \
            [new(T, B, m + 2 * N) for _ in range(kept)]
        p.u, p.s = [new(T, B, m) for _ in range(kept)], [new(T, B, m) for _ in range(kept)]
        p.o = [new(T, B, n) for _ in range(kept)]
        v, z = p.vz[0].split(m, dim=2)
        d, b, c = self._vectors(p.dbc[0])
        p.conv = snn.shortconv_desc(v, p.u[0], self.taps, "silu")
        p.scan = snn.selscan_desc(p.u[0], d, b, c, p.s[0], z, forward_only=not train)
        p.pre = snn.layer_norm_desc(p.x[0], p.h[0], self.eps)
        p.post = snn.gate_norm_desc(p.x[0], p.o[0], None, 1, "none", self.eps)
        denses = (p.embed, p.readout, p.w_in, p.w_x, p.w_out)
        sizes = [snn.snn_layer_workspace_bytes(d) for d in denses]
        sizes += [snn.snn_selscan_workspace_bytes(p.scan)]
        p.saved = [None] * L
        if train:
            sizes += [snn.snn_shortconv_workspace_bytes(p.conv),
                      snn.snn_layer_norm_workspace_bytes(p.pre),
                      snn.snn_gate_norm_workspace_bytes(p.post),
                      snn.snn_loss_workspace_bytes(snn.LOSS_CE_COUNT, B, self.n_out)]
            p.saved = [new(max(16, snn.snn_selscan_saved_bytes(p.scan)), dtype=torch.uint8)
                       for _ in range(L)]
            p.spk = new(T, B, self.n_out, dtype=torch.uint8)
            p.kept = new(snn.snn_layer_saved_bytes(p.readout), dtype=torch.uint8)
            p.counts, p.gcounts = new(B, self.n_out), new(B, self.n_out)
            p.dx, p.dh, p.do = new(T, B, n), new(T, B, n), new(T, B, n)
            p.dvz, p.ddbc = new(T, B, 2 * m), new(T, B, m + 2 * N)
            p.du, p.ds, p.du_x = new(T, B, m), new(T, B, m), new(T, B, m)
            p.da = new(N, m)
        p.ws = new(max(sizes + [256]), dtype=torch.uint8)
        p.bytes = sum(t.numel() * t.element_size() for t in p.bufs)
        return p

    def _vectors(self, dbc):
        """Raw steps [T,B,width], b and c [T,B,1,states] of a packed projection."""
        N = self.n_states
        d, b, c = dbc.split([self.width, N, N], dim=2)
        return d, b.unsqueeze(2), c.unsqueeze(2)

    def states(self, n):
        """Zero states of n sequences (or request slots): per block the convolution's last
        inputs and the scan's integrators."""
        zeros = self.torch.zeros
        return [(zeros((n, self.taps - 1, self.width), device=self.device),
                 zeros((n, self.n_states, self.width), device=self.device)) for _ in self.W]

    # ---- forward -------------------------------------------------------------
    def _blocks(self, p, spikes, conv, scan):
        """Embedding and blocks; conv(block, v, u) and scan(block, inputs, s) run their
        operators."""
        at = (lambda a, i: a[i % len(a)])
        snn.snn_synapse_fwd(p.embed, spikes, self.E, None, p.x[0], None, p.ws)
        for i in range(len(self.W)):
            x, h, vz, dbc = at(p.x, i), at(p.h, i), at(p.vz, i), at(p.dbc, i)
            u, s, o = at(p.u, i), at(p.s, i), at(p.o, i)
            snn.snn_layer_norm_fwd(p.pre, x, self.ln_w[i], self.ln_b[i], h)
            snn.snn_synapse_fwd(p.w_in, h, self.W[i], None, vz, None, p.ws)
            v, z = vz.split(self.width, dim=2)
            conv(i, v, u)
            snn.snn_synapse_fwd(p.w_x, u, self.W_x[i], None, dbc, None, p.ws)
            d, b, c = self._vectors(dbc)
            scan(i, (u, d, -self.log_a[i].exp(), b, c, self.skip[i], self.dt_bias[i], z), s)
            snn.snn_synapse_fwd(p.w_out, s, self.W_out[i], None, o, None, p.ws)
            snn.snn_gate_norm_fwd(p.post, x, o, None, self.w_post[i], self.scale[i], None,
                                  at(p.x, i + 1), None)
        L = len(self.W)
        snn.snn_layer_norm_fwd(p.pre, at(p.x, L), self.ln_w[L], self.ln_b[L], at(p.h, L))
        return at(p.h, L)

    def prompt(self, spikes, states, lens=None):
        """Whole sequences spikes [T,B,n_in] u8 from `states` (updated in place); returns
        the readout's currents [T,B,n_out], a tensor of their own.  lens: int32 [B]."""
        T, B = spikes.shape[:2]
        spikes, p = self._spikes(spikes, T, B), self._plan(T, B)

        def conv(i, v, u):
            snn.snn_shortconv_fwd(p.conv, v, self.conv_w[i], self.conv_b[i], lens, states[i][0], u,
                                  states[i][0])

        def scan(i, ins, s):
            snn.snn_selscan_fwd(p.scan, *ins, lens, states[i][1], s, states[i][1], None, p.ws)

        return self._currents(p, self._blocks(p, spikes, conv, scan))

    def step(self, spikes, states, slots=None):
        """One time step spikes [B,n_in] of running requests; request b's states lie in slot
        slots[b] (int32, or b), updated in place.  Returns the currents [B,n_out]."""
        B = spikes.shape[0]
        spikes, p = self._spikes(spikes.unsqueeze(0), 1, B), self._plan(1, B)

        def conv(i, v, u):
            snn.snn_shortconv_step(p.conv, v, self.conv_w[i], self.conv_b[i], slots, states[i][0],
                                   states[i][0], u)

        def scan(i, ins, s):
            snn.snn_selscan_step(p.scan, *ins, slots, states[i][1], states[i][1], s)

        return self._currents(p, self._blocks(p, spikes, conv, scan))[0]

    # ---- training ------------------------------------------------------------
    def train_step(self, spikes, labels):
        """Forward, cross-entropy on the readout's spike counts, and backward: gradients in
        ``grads`` (of ``params``), the loss in the returned tensor.  spikes [T,B,n_in] u8,
        labels int32 [B]."""
        B, L, m = self.B, len(self.W), self.width
        spikes, labels = self._spikes(spikes, self.T, B), self._labels(labels, B)
        p = self._plan(self.T, B, True)
        ins = [None] * L

        def conv(i, v, u):
            snn.snn_shortconv_fwd(p.conv, v, self.conv_w[i], self.conv_b[i], None, None, u, None)

        def scan(i, args, s):
            ins[i] = args
            snn.snn_selscan_fwd(p.scan, *args, None, None, s, None, p.saved[i], p.ws)

        h = self._blocks(p, spikes, conv, scan)
        snn.snn_layer_fwd(p.readout, h, self.R, None, None, p.spk, p.kept, p.counts, p.ws)
        loss = h.new_empty(4)
        snn.snn_loss(snn.LOSS_CE_COUNT, B, self.n_out, 1, p.counts, labels, None, loss,
                     p.gcounts, p.ws)
        snn.snn_layer_bwd(p.readout, snn.GRAD_BCAST, p.gcounts, h, self.R, None, p.kept, self.g_R,
                          None, None, p.dh, p.ws)
        snn.snn_layer_norm_bwd(p.pre, p.x[L], p.dh, None, self.ln_w[L], p.dx, self.g_ln_w[L],
                               self.g_ln_b[L], p.ws)
        dv, dz = p.dvz.split(m, dim=2)
        dd, db, dc = self._vectors(p.ddbc)
        for i in reversed(range(L)):  # p.dx: the gradient of x[i + 1], then of x[i]
            v = p.vz[i].split(m, dim=2)[0]
            snn.snn_gate_norm_bwd(p.post, p.dx, None, None, p.o[i], None, None, None,
                                  self.w_post[i], self.scale[i], None, p.dx, p.do, None,
                                  self.g_w_post[i], self.g_scale[i], None, p.ws)
            snn.snn_synapse_bwd(p.w_out, p.do, None, p.s[i], self.W_out[i], self.g_W_out[i], p.ds,
                                p.ws)
            snn.snn_selscan_bwd(p.scan, *ins[i], None, p.saved[i], p.ds, None, p.du, dd, p.da, db,
                                dc, self.g_skip[i], self.g_dt_bias[i], dz, None, p.ws)
            self.torch.mul(p.da, ins[i][2], out=self.g_log_a[i])
            snn.snn_synapse_bwd(p.w_x, p.ddbc, None, p.u[i], self.W_x[i], self.g_W_x[i], p.du_x,
                                p.ws)
            p.du.add_(p.du_x)
            snn.snn_shortconv_bwd(p.conv, v, self.conv_w[i], self.conv_b[i], None, None, p.du, None,
                                  dv, self.g_conv_w[i], self.g_conv_b[i], None, p.ws)
            snn.snn_synapse_bwd(p.w_in, p.dvz, None, p.h[i], self.W[i], self.g_W[i], p.dh, p.ws)
            snn.snn_layer_norm_bwd(p.pre, p.x[i], p.dh, p.dx, self.ln_w[i], p.dx, self.g_ln_w[i],
                                   self.g_ln_b[i], p.ws)
        snn.snn_synapse_bwd(p.embed, p.dx, None, spikes, self.E, self.g_E, None, p.ws)
        return loss[0]


def main():
    import torch
    T, B, n_in, classes = 100, 64, 96, 4
    net = SelectiveNet(n_in, n=128, width=256, states=16, blocks=2, n_out=classes, T=T, B=B)
    net.init_adamw(lr=5e-4)
    for i in range(200):
        x, y = (torch.as_tensor(a).cuda() for a in spike_trains(T, B, n_in, classes, seed=i))
        loss = net.train_step(x, y)
        net.update()
        if i % 20 == 19:
            print(f"step {i:3d}  loss {loss.item():.4f}", flush=True)
    # a prompt of 60 steps, then the rest one by one, against the whole sequence
    states, whole = net.states(B), net.states(B)
    want = net.prompt(x, whole)
    net.prompt(x[:60].contiguous(), states)
    err = max((net.step(x[t], states) - want[t]).abs().max().item() for t in range(60, T))
    print(f"currents step by step against the whole prompt: {err:.2e}", flush=True)


if __name__ == "__main__":
    main()
