"""A sequence model of leaky blocks on spike trains: the block operators together.

    x0  = E spikes_t                                   one dense synapse per step
    per block:  q | k | v | gate = W norm(x)           one dense synapse
                o   = linear attention of q, k, v with a decay per head
                x   = x + scale norm_per_head(o) w_post silu(gate)
    readout:    Leaky neurons on norm(x), loss on their spike counts

The state of a block leaks as the neurons' membranes do (S_t = g S_{t-1} +
k_t^T v_t), so whole sequences train and run in parallel over time, and single
steps go on from the states alone.  Everything is fp32 and runs in the
library; torch holds the memory.

``python -m paper_2211_10725_amd.sequence`` trains one on synthetic spike trains
and continues a prompt step by step.
"""
from __future__ import annotations

import numpy as np

import paper_2211_10725_amd as snn


class SequenceNet:
    """Parameters, buffers and call sequence of the model above.

    n_in inputs, `heads` heads of d_v values (the residual stream's width is
    heads * d_v), kv_heads key and value heads, `blocks` blocks, n_out output
    neurons.  checkpoints: what the backward needs of a block (its attention
    output and gate, its q, k, v and its normed input) is held in 8 bits between
    the passes, in one fourth of the memory; the gradients are then taken at the
    values those stand for."""

    def __init__(self, n_in, heads, kv_heads, d_k, d_v, blocks, n_out, T, B, beta=0.5,
                 slope=3.0, checkpoints=False, eps=1e-6, seed=0, device="cuda"):
        import torch
        self.torch, self.device = torch, device
        self.T, self.B, self.heads, self.kv_heads = T, B, heads, kv_heads
        self.d_k, self.d_v, self.eps, self.checkpoints = d_k, d_v, eps, checkpoints
        self.n, self.n_in, self.n_out = heads * d_v, n_in, n_out
        self.beta, self.slope = beta, slope
        self.widths = [heads * d_k, kv_heads * d_k, kv_heads * d_v, self.n]
        self.n_qkv, self.n_proj = sum(self.widths[:3]), sum(self.widths)
        # one scale never spans two heads: the norm per head would magnify what a
        # large neighbour leaves of a small head's digits
        self.block = min(128, d_v & -d_v)
        self.qkv_block = min(128, d_k & -d_k, d_v & -d_v)
        rng = np.random.default_rng(seed)

        def uniform(rows, cols):
            a = rng.uniform(-1, 1, (rows, cols)) / np.sqrt(cols)
            return torch.as_tensor(a, dtype=torch.float32).to(device)

        def ones(v=1.0):
            return torch.full((self.n,), v, dtype=torch.float32, device=device)

        # decays 1 - 2^-1 .. 1 - 2^-7: memories of 2 to 128 steps
        g = 1 - 2.0 ** -np.linspace(1, 7, heads)
        self.decay = torch.as_tensor(g, dtype=torch.float32).to(device)
        self.E = uniform(self.n, n_in)
        self.W = [uniform(self.n_proj, self.n) for _ in range(blocks)]
        self.w_pre = [ones() for _ in range(blocks + 1)]
        self.w_post, self.scale = [ones() for _ in range(blocks)], [ones(0.5) for _ in range(blocks)]
        self.R = uniform(n_out, self.n)
        self.params = [self.E, *self.W, *self.w_pre, *self.w_post, *self.scale, self.R]
        self.grads = [torch.empty_like(p) for p in self.params]
        it = iter(self.grads)
        self.gE = next(it)
        self.gW = [next(it) for _ in self.W]
        self.gw_pre = [next(it) for _ in self.w_pre]
        self.gw_post = [next(it) for _ in self.w_post]
        self.gscale = [next(it) for _ in self.scale]
        self.gR = next(it)
        self.plans = {}

    # ---- buffers and descriptors of one shape -------------------------------
    def _plan(self, T, B, train=False):
        """Descriptors and buffers for T steps of B sequences (`train`: with what
        the backward needs), kept for later calls of the shape.  Those of prompts
        and steps hold at most four times the largest's memory together: the
        longest unused go first, but never one that a graph was captured from."""
        key = (T, B, train)
        p = self.plans.pop(key, None)
        made = p is None
        if made:
            p = self._new_plan(T, B, train)
        self.plans[key] = p  # the last one used is the last
        if p.stream is not None:
            stream = snn._stream(None)
            if stream != p.stream and stream not in p.others:
                p.others[stream] = self.torch.cuda.current_stream()
            p.stays = p.stays or self.torch.cuda.is_current_stream_capturing()
        if made:
            self._drop_plans(p)
        return p

    def _drop_plans(self, newest):
        old = {k: p for k, p in self.plans.items() if not k[2] and not p.stays}
        held = [p.bytes for p in old.values()]
        most, held, count = 4 * max(held, default=0), sum(held), len(held)
        for k, p in old.items():
            if (held <= most and count <= 256) or p is newest:
                break
            del self.plans[k]
            held, count = held - p.bytes, count - 1
            for t in p.bufs:  # their memory is free once those streams are done, too
                for other in p.others.values():
                    t.record_stream(other)

    def _new_plan(self, T, B, train):
        torch = self.torch
        p = type("Plan", (), {})()
        p.bufs, p.others, p.stays = [], {}, False
        p.stream = snn._stream(None) if torch.device(self.device).type == "cuda" else None
        L = len(self.W)

        def new(*shape, dtype):
            p.bufs.append(torch.empty(shape, dtype=dtype, device=self.device))
            return p.bufs[-1]

        def buf(*shape):
            return new(*shape, dtype=torch.float32)

        def dense(n_in, n_out, in_dtype=snn.F32):
            return snn.layer_desc(dict(kind="dense", n_in=n_in, n_out=n_out, neuron="leaky",
                                       beta=self.beta), T, B, in_dtype=in_dtype, slope=self.slope)

        p.embed, p.proj, p.readout = (dense(self.n_in, self.n, snn.U8),
                                      dense(self.n, self.n_proj), dense(self.n, self.n_out))
        kept = L if train and not self.checkpoints else 1
        p.x = [buf(T, B, self.n) for _ in range(L + 1 if train else 2)]
        p.h = [buf(T, B, self.n) for _ in range(L + 1 if kept == L else 2)]
        p.cur = [buf(T, B, self.n_proj) for _ in range(kept)]
        p.o = [buf(T, B, self.n) for _ in range(kept)]
        q, k, v, gate = self._parts(p.cur[0])
        o = p.o[0].unflatten(2, (self.heads, self.d_v))
        p.attn = snn.linattn_desc(q, k, v, o, forward_only=not train)
        p.norm = snn.gate_norm_desc(p.x[0], p.o[0], gate, self.heads, "silu", self.eps,
                                    ckpt_block=self.block)
        p.first = snn.gate_norm_desc(p.x[0], None, None, 1, "none", self.eps)
        sizes = [snn.snn_layer_workspace_bytes(d) for d in (p.embed, p.proj, p.readout)]
        sizes += [snn.snn_linattn_workspace_bytes(p.attn)]
        if train:
            sizes += [snn.snn_gate_norm_workspace_bytes(d) for d in (p.norm, p.first)]
            sizes += [snn.snn_loss_workspace_bytes(snn.LOSS_CE_COUNT, B, self.n_out)]
            p.spk = new(T, B, self.n_out, dtype=torch.uint8)
            p.saved = new(snn.snn_layer_saved_bytes(p.readout), dtype=torch.uint8)
            p.counts, p.gcounts = buf(B, self.n_out), buf(B, self.n_out)
            p.dx, p.dh, p.dcur = buf(T, B, self.n), buf(T, B, self.n), buf(T, B, self.n_proj)
            p.do = buf(T, B, self.n)
            if self.checkpoints:
                def ckpt(n, block):
                    return [new(snn.snn_checkpoint_bytes(T * B, n, block), dtype=torch.uint8)
                            for _ in range(L)]
                p.o8, p.gate8 = ckpt(self.n, self.block), ckpt(self.n, self.block)
                p.h8, p.qkv8 = ckpt(self.n, 128), ckpt(self.n_qkv, self.qkv_block)
        p.ws = new(max(sizes + [256]), dtype=torch.uint8)
        p.bytes = sum(t.numel() * t.element_size() for t in p.bufs)
        return p

    def _parts(self, cur):
        """q, k, v by heads and the gate of a packed projection."""
        q, k, v, gate = cur.split(self.widths, dim=2)
        return (q.unflatten(2, (-1, self.d_k)), k.unflatten(2, (-1, self.d_k)),
                v.unflatten(2, (-1, self.d_v)), gate)

    def states(self, n):
        """Zero states of n sequences (or request slots), one tensor per block."""
        return [self.torch.zeros((n, self.heads, self.d_k, self.d_v), device=self.device)
                for _ in self.W]

    # ---- forward -------------------------------------------------------------
    def _run(self, p, spikes, attend, train):
        """Embedding and blocks; attend(block, q, k, v, o) runs the attention."""
        L = len(self.W)
        at = (lambda a, i: a[i % len(a)])
        snn.snn_synapse_fwd(p.embed, spikes, self.E, None, p.x[0], None, p.ws)
        snn.snn_gate_norm_fwd(p.first, p.x[0], None, None, None, None, self.w_pre[0], None, p.h[0])
        for i in range(L):
            h, cur, o = at(p.h, i), at(p.cur, i), at(p.o, i)
            snn.snn_synapse_fwd(p.proj, h, self.W[i], None, cur, None, p.ws)
            q, k, v, gate = self._parts(cur)
            attend(i, q, k, v, o.unflatten(2, (self.heads, self.d_v)))
            ckpt = train and self.checkpoints
            if ckpt:
                snn.snn_checkpoint_save(h, p.h8[i])
                snn.snn_checkpoint_save(cur[:, :, :self.n_qkv], p.qkv8[i], self.qkv_block)
            snn.snn_gate_norm_fwd(p.norm, at(p.x, i), o, gate, self.w_post[i], self.scale[i],
                                  self.w_pre[i + 1], at(p.x, i + 1), at(p.h, i + 1),
                                  p.o8[i] if ckpt else None, p.gate8[i] if ckpt else None)
        return at(p.h, L)

    def _currents(self, p, h):
        out = h.new_empty((*h.shape[:2], self.n_out))
        snn.snn_synapse_fwd(p.readout, h, self.R, None, out, None, p.ws)
        return out

    def prompt(self, spikes, states, lens=None):
        """Whole sequences spikes [T,B,n_in] u8 from `states` (updated in place);
        returns the readout's currents [T,B,n_out], a tensor of their own.  lens:
        int32 [B] lengths."""
        T, B = spikes.shape[:2]
        p = self._plan(T, B)

        def attend(i, q, k, v, o):
            snn.snn_linattn_fwd(p.attn, q, k, v, self.decay, lens, states[i], o, states[i], p.ws)

        return self._currents(p, self._run(p, spikes, attend, False))

    def step(self, spikes, states, slots=None):
        """One time step spikes [B,n_in] of running requests; request b's states
        lie in slot slots[b] (int32, or b) of `states`, updated in place.  Returns
        the currents [B,n_out]."""
        B = spikes.shape[0]
        p = self._plan(1, B)

        def attend(i, q, k, v, o):
            snn.snn_linattn_step(p.attn, q, k, v, self.decay, slots, states[i], states[i], o)

        return self._currents(p, self._run(p, spikes.unsqueeze(0), attend, False))[0]

    # ---- training ------------------------------------------------------------
    def train_step(self, spikes, labels):
        """Forward, cross-entropy on the readout's spike counts, and backward:
        gradients in ``grads`` (of ``params``), the loss in the returned tensor."""
        T, B, L = self.T, self.B, len(self.W)
        p = self._plan(T, B, True)

        def attend(i, q, k, v, o):
            snn.snn_linattn_fwd(p.attn, q, k, v, self.decay, None, None, o, None, p.ws)

        h = self._run(p, spikes, attend, True)
        snn.snn_layer_fwd(p.readout, h, self.R, None, None, p.spk, p.saved, p.counts, p.ws)
        loss = h.new_empty(4)
        snn.snn_loss(snn.LOSS_CE_COUNT, B, self.n_out, 1, p.counts, labels, None, loss,
                     p.gcounts, p.ws)
        snn.snn_layer_bwd(p.readout, snn.GRAD_BCAST, p.gcounts, h, self.R, None, p.saved, self.gR,
                          None, None, p.dh, p.ws)
        heads = (self.heads, self.d_v)
        dq, dk, dv, dgate = self._parts(p.dcur)
        for i in reversed(range(L)):
            if self.checkpoints:
                h, cur, o, gate = p.h[0], p.cur[0], None, None
                kept = (p.o8[i], p.gate8[i])
            else:
                h, cur, o, kept = p.h[i], p.cur[i], p.o[i], (None, None)
                gate = self._parts(cur)[3]
            # p.dx holds the gradient of x[i + 1] from the blocks above (none at the top)
            snn.snn_gate_norm_bwd(p.norm, p.dx if i + 1 < L else None, p.dh, p.x[i + 1], o, gate,
                                  *kept, self.w_post[i], self.scale[i], self.w_pre[i + 1], p.dx,
                                  p.do, dgate, self.gw_post[i], self.gscale[i],
                                  self.gw_pre[i + 1], p.ws)
            if self.checkpoints:
                snn.snn_checkpoint_load(p.h8[i], h)
                snn.snn_checkpoint_load(p.qkv8[i], cur[:, :, :self.n_qkv], self.qkv_block)
            q, k, v, _ = self._parts(cur)
            snn.snn_linattn_bwd(p.attn, q, k, v, self.decay, None, None, p.do.unflatten(2, heads),
                                None, dq, dk, dv, None, p.ws)
            snn.snn_synapse_bwd(p.proj, p.dcur, None, h, self.W[i], self.gW[i], p.dh, p.ws)
        snn.snn_gate_norm_bwd(p.first, p.dx, p.dh, p.x[0], None, None, None, None, None, None,
                              self.w_pre[0], p.dx, None, None, None, None, self.gw_pre[0], p.ws)
        snn.snn_synapse_bwd(p.embed, p.dx, None, spikes, self.E, self.gE, None, p.ws)
        return loss[0]

    def init_adamw(self, **hparams):
        zeros = self.torch.zeros_like
        self.opt, self.opt_t = hparams, 0
        self.moments = [(zeros(p), zeros(p)) for p in self.params]

    def update(self):
        """One AdamW step with the gradients of the last ``train_step``."""
        self.opt_t += 1
        snn.snn_adamw([(p, g, m, v, None) for p, g, (m, v) in
                       zip(self.params, self.grads, self.moments)], self.opt_t, **self.opt)


def spike_trains(T, B, n_in, classes, seed=0):
    """Sequences whose class is the order in which two halves of the inputs fire
    faster: labels int32 [B], spikes u8 [T,B,n_in]."""
    rng = np.random.default_rng(seed)
    y = rng.integers(0, classes, B)
    phase = (np.arange(T)[:, None] * classes // T == y[None]).astype(float)  # [T,B]
    fast = np.arange(n_in) < n_in // 2
    rate = np.where(fast, 0.05 + 0.4 * phase[:, :, None], 0.15)
    return (rng.random((T, B, n_in)) < rate).astype(np.uint8), y.astype(np.int32)


def main():
    import torch
    T, B, n_in, classes = 100, 64, 96, 4
    net = SequenceNet(n_in, heads=4, kv_heads=2, d_k=32, d_v=32, blocks=2, n_out=classes, T=T, B=B,
                      checkpoints=True)
    net.init_adamw(lr=1e-3)
    for i in range(100):
        x, y = (torch.as_tensor(a).cuda() for a in spike_trains(T, B, n_in, classes, seed=i))
        loss = net.train_step(x, y)
        net.update()
        if i % 10 == 9:
            print(f"step {i:3d}  loss {loss.item():.4f}", flush=True)
    # a prompt of 60 steps, then the rest one by one, against the whole sequence
    states, whole = net.states(B), net.states(B)
    want = net.prompt(x, whole).clone()
    net.prompt(x[:60].contiguous(), states)
    err = max((net.step(x[t], states) - want[t]).abs().max().item() for t in range(60, T))
    print(f"currents step by step against the whole prompt: {err:.2e}", flush=True)


if __name__ == "__main__":
    main()
