"""MI355X-native spiking-layer training: time-stepped forward and BPTT backward.

Thin ctypes binding over ``libsnn.so`` (C ABI declared in ``include/snn.h``).
The functions below have the ABI's names and only marshal arguments: torch
tensors supply device pointers and the HIP stream, every step of the method
runs in the library's HIP kernels.  There is no CPU fallback: if the library
is missing, the first call raises.

``Network`` chains the layer calls of a feed-forward spiking network (layers
ascending in the forward pass, loss on the output spike counts, layers
descending in the backward pass), the training step the paper times
(Sec. IV "Baseline Throughput", without the optimizer update).
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

from . import workloads  # noqa: F401  (seeded inputs; no method arithmetic)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsnn.so")

# element types, neuron models, synapses, gradient kinds, losses (snn.h)
F32, F16, BF16, U8 = 0, 1, 2, 3
SPK_BITS = 4  # spikes packed 64 to a word (an output type only)
LEAKY, SYNAPTIC, RLEAKY = 0, 1, 2
SYN_DENSE, SYN_CONV5_POOL2, SYN_NONE = 0, 1, 2
RESET_DETACHED, RESET_SURROGATE = 0, 1
GRAD_FULL, GRAD_BCAST, GRAD_FOLD = 0, 1, 2
LOSS_CE_COUNT, LOSS_MSE_COUNT = 0, 1
FLAG_FP32_MFMA = 1
ABI_VERSION = 14
DCUR_T_TRANSPOSED, DCUR_T_PLANES = 1, 2
GATE_NONE, GATE_MUL, GATE_SIGMOID, GATE_SILU = 0, 1, 2, 3

STATUS = {0: "SNN_OK", 1: "SNN_ERR_NULL", 2: "SNN_ERR_SHAPE", 3: "SNN_ERR_DTYPE",
          4: "SNN_ERR_ALIGN", 5: "SNN_ERR_UNSUPPORTED", 6: "SNN_ERR_WORKSPACE",
          7: "SNN_ERR_HIP"}

EXPORTS = ["snn_abi_version", "snn_status_str", "snn_layer_saved_bytes",
           "snn_layer_workspace_bytes", "snn_layer_fwd", "snn_layer_bwd",
           "snn_loss_workspace_bytes", "snn_loss", "snn_synapse_fwd", "snn_neuron_fwd",
           "snn_neuron_bwd", "snn_synapse_bwd", "snn_adamw", "snn_loss_noalloc",
           "snn_layer_saved_layout", "snn_layer_dcur_t_bytes", "snn_layer_dcur_t_layout",
           "snn_fused_step_check", "snn_fused_step_workspace_bytes", "snn_fused_step",
           "snn_linattn_workspace_bytes", "snn_linattn_fwd", "snn_linattn_bwd",
           "snn_linattn_step", "snn_gate_norm_workspace_bytes", "snn_gate_norm_fwd",
           "snn_gate_norm_bwd", "snn_checkpoint_bytes", "snn_checkpoint_save",
           "snn_checkpoint_load", "snn_selscan_saved_bytes", "snn_selscan_workspace_bytes",
           "snn_selscan_fwd", "snn_selscan_bwd", "snn_selscan_step",
           "snn_shortconv_workspace_bytes", "snn_shortconv_fwd", "snn_shortconv_bwd",
           "snn_shortconv_step", "snn_layer_norm_workspace_bytes", "snn_layer_norm_fwd",
           "snn_layer_norm_bwd"]


class LayerDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("B", ctypes.c_int32),
                ("synapse", ctypes.c_int32), ("neuron", ctypes.c_int32),
                ("n_in", ctypes.c_int32), ("n_out", ctypes.c_int32),
                ("c_in", ctypes.c_int32), ("h_in", ctypes.c_int32),
                ("w_in", ctypes.c_int32), ("c_out", ctypes.c_int32),
                ("in_dtype", ctypes.c_int32), ("w_dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("reset_grad", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("beta", ctypes.c_float), ("alpha", ctypes.c_float),
                ("threshold", ctypes.c_float), ("slope", ctypes.c_float)]

    def copy(self):
        d = LayerDesc()
        ctypes.pointer(d)[0] = self
        return d


class SavedLayout(ctypes.Structure):
    _fields_ = [("bytes", ctypes.c_size_t), ("cur_offset", ctypes.c_size_t),
                ("cur_bytes", ctypes.c_size_t), ("ckpt_offset", ctypes.c_size_t),
                ("ckpt_bytes", ctypes.c_size_t), ("pool_offset", ctypes.c_size_t),
                ("pool_bytes", ctypes.c_size_t), ("ckpt_interval", ctypes.c_int32),
                ("ckpt_count", ctypes.c_int32), ("ckpt_planes", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class FusedDesc(ctypes.Structure):
    _fields_ = [("hidden", LayerDesc), ("readout", LayerDesc), ("loss_kind", ctypes.c_int32),
                ("pop", ctypes.c_int32), ("wait_limit", ctypes.c_uint32),
                ("reserved", ctypes.c_int32)]


class GradIn(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("n_up", ctypes.c_int32),
                ("g", ctypes.c_void_p), ("dcur_up", ctypes.c_void_p), ("w_up", ctypes.c_void_p),
                ("dcur_up_dtype", ctypes.c_int32), ("w_up_dtype", ctypes.c_int32)]


class AdamwTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("param_half", ctypes.c_void_p), ("n", ctypes.c_int64)]


class AdamwHparams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float),
                ("step", ctypes.c_int32)]


class LinattnDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("B", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("d_k", ctypes.c_int32), ("d_v", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3),
                ("forward_only", ctypes.c_int32)]


class GateNormDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("n", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("gate", ctypes.c_int32), ("x_dtype", ctypes.c_int32),
                ("y_dtype", ctypes.c_int32), ("eps", ctypes.c_float),
                ("ckpt_block", ctypes.c_int32), ("ld_x", ctypes.c_int64),
                ("ld_y", ctypes.c_int64), ("ld_g", ctypes.c_int64), ("ld_h", ctypes.c_int64)]


class SelscanDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("B", ctypes.c_int32), ("n", ctypes.c_int32),
                ("states", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("delta_softplus", ctypes.c_int32),
                ("forward_only", ctypes.c_int32), ("u_stride", ctypes.c_int64 * 2),
                ("dt_stride", ctypes.c_int64 * 2), ("z_stride", ctypes.c_int64 * 2),
                ("y_stride", ctypes.c_int64 * 2), ("b_stride", ctypes.c_int64 * 3),
                ("c_stride", ctypes.c_int64 * 3)]


class ShortconvDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("B", ctypes.c_int32), ("n", ctypes.c_int32),
                ("width", ctypes.c_int32), ("act", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("x_stride", ctypes.c_int64 * 2), ("y_stride", ctypes.c_int64 * 2)]


class LayerNormDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("n", ctypes.c_int32), ("x_dtype", ctypes.c_int32),
                ("y_dtype", ctypes.c_int32), ("eps", ctypes.c_float), ("ld_x", ctypes.c_int64),
                ("ld_y", ctypes.c_int64)]


class SNNError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__(f"{fn} failed: {STATUS.get(status, status)} "
                         f"({_lib.snn_status_str(status).decode() if _lib else ''})")


_lib = None


def lib():
    """Load libsnn.so (built in-tree by ``build.build()``); raise if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"HIP library {LIB_PATH} is not built; run __graft_entry__.build()")
    L = ctypes.CDLL(LIB_PATH)
    P, S = ctypes.c_void_p, ctypes.c_size_t
    D = ctypes.POINTER(LayerDesc)
    G = ctypes.POINTER(GradIn)
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    LA, GN = ctypes.POINTER(LinattnDesc), ctypes.POINTER(GateNormDesc)
    SS, SC, LN = (ctypes.POINTER(d) for d in (SelscanDesc, ShortconvDesc, LayerNormDesc))
    sig = {
        "snn_abi_version": ([], ctypes.c_int),
        "snn_status_str": ([ctypes.c_int], ctypes.c_char_p),
        "snn_layer_saved_bytes": ([D], S),
        "snn_layer_saved_layout": ([D, ctypes.POINTER(SavedLayout)], ctypes.c_int),
        "snn_layer_workspace_bytes": ([D], S),
        "snn_layer_fwd": ([D, P, P, P, P, P, P, P, P, S, P], ctypes.c_int),
        "snn_layer_bwd": ([D, G, P, P, P, P, P, P, P, P, P, S, P], ctypes.c_int),
        "snn_loss_workspace_bytes": ([i32, i32, i32], S),
        "snn_loss": ([i32, i32, i32, i32, P, P, P, P, P, P, S, P], ctypes.c_int),
        "snn_loss_noalloc": ([i32, i32, i32, i32, P, P, P, P, P, P], ctypes.c_int),
        "snn_synapse_fwd": ([D, P, P, P, P, P, P, S, P], ctypes.c_int),
        "snn_neuron_fwd": ([D, P, P, P, P, P, P, P], ctypes.c_int),
        "snn_neuron_bwd": ([D, G, P, P, P, P, P, P, P, P, P, S, P], ctypes.c_int),
        "snn_synapse_bwd": ([D, P, P, P, P, P, P, P, P, P, S, P], ctypes.c_int),
        "snn_layer_dcur_t_bytes": ([D], S),
        "snn_layer_dcur_t_layout": ([D], i32),
        "snn_fused_step_check": ([ctypes.POINTER(FusedDesc)], ctypes.c_int),
        "snn_fused_step_workspace_bytes": ([ctypes.POINTER(FusedDesc)], S),
        "snn_fused_step": ([ctypes.POINTER(FusedDesc)] + [P] * 16 + [S, P], ctypes.c_int),
        "snn_adamw": ([ctypes.POINTER(AdamwTensor), i32, ctypes.POINTER(AdamwHparams), P],
                      ctypes.c_int),
        "snn_linattn_workspace_bytes": ([LA], S),
        "snn_linattn_fwd": ([LA] + [P] * 9 + [S, P], ctypes.c_int),
        "snn_linattn_bwd": ([LA] + [P] * 13 + [S, P], ctypes.c_int),
        "snn_linattn_step": ([LA] + [P] * 5 + [i32] + [P] * 4, ctypes.c_int),
        "snn_gate_norm_workspace_bytes": ([GN], S),
        "snn_gate_norm_fwd": ([GN] + [P] * 11, ctypes.c_int),
        "snn_gate_norm_bwd": ([GN] + [P] * 17 + [S, P], ctypes.c_int),
        "snn_checkpoint_bytes": ([i32, i32, i32], S),
        "snn_checkpoint_save": ([i32, i32, i32, i64, i32, P, P, P], ctypes.c_int),
        "snn_checkpoint_load": ([i32, i32, i32, i64, i32, P, P, P], ctypes.c_int),
        "snn_selscan_saved_bytes": ([SS], S),
        "snn_selscan_workspace_bytes": ([SS], S),
        "snn_selscan_fwd": ([SS] + [P] * 14 + [S, P], ctypes.c_int),
        "snn_selscan_bwd": ([SS] + [P] * 22 + [S, P], ctypes.c_int),
        "snn_selscan_step": ([SS] + [P] * 9 + [i32] + [P] * 4, ctypes.c_int),
        "snn_shortconv_workspace_bytes": ([SC], S),
        "snn_shortconv_fwd": ([SC] + [P] * 8, ctypes.c_int),
        "snn_shortconv_bwd": ([SC] + [P] * 12 + [S, P], ctypes.c_int),
        "snn_shortconv_step": ([SC] + [P] * 4 + [i32] + [P] * 4, ctypes.c_int),
        "snn_layer_norm_workspace_bytes": ([LN], S),
        "snn_layer_norm_fwd": ([LN] + [P] * 5, ctypes.c_int),
        "snn_layer_norm_bwd": ([LN] + [P] * 8 + [S, P], ctypes.c_int),
    }
    for name, (args, res) in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res
    if L.snn_abi_version() != ABI_VERSION:
        raise RuntimeError("libsnn.so ABI version mismatch")
    _lib = L
    return L


# --------------------------------------------------------------------------
# argument marshalling
# --------------------------------------------------------------------------
def _p(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def _stream(stream):
    if stream is None:
        import torch
        if torch.cuda.is_initialized():
            # the current stream's handle itself: a Stream object around it costs
            # several microseconds, more than a small call's kernel
            try:
                return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
            except AttributeError:  # torch's private names
                pass
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(fn, st):
    if st != 0:
        raise SNNError(fn, st)


def _dtype_code(t):
    import torch
    return {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}[t.dtype]


def _grad_in(kind, g):
    """The upstream gradient argument: g a tensor for GRAD_FULL / GRAD_BCAST,
    or (dcur_up, w_up) for GRAD_FOLD (dL/dI [T,B,n_up] and the weights
    [n_up, n_out] of the dense layer above)."""
    if kind == GRAD_FOLD:
        dup, wup = g
        return GradIn(kind, int(wup.shape[0]), None, _p(dup), _p(wup), _dtype_code(dup),
                      _dtype_code(wup))
    return GradIn(kind, 0, _p(g), None, None, 0, 0)


I32 = 100  # int32 arguments (labels, status): not a layer dtype
_ELEM = {F32: 4, F16: 2, BF16: 2, U8: 1, I32: 4}


def _need(fn, t, dtype_code, count, what):
    """A tensor argument must hold at least `count` elements of the type the
    descriptor names (the library cannot see buffer sizes): raise before the
    call instead of letting a kernel run past the buffer."""
    if t is None or isinstance(t, int):
        return
    es = _ELEM[dtype_code]
    if t.element_size() != es or t.numel() < count:
        raise ValueError(f"{fn}: {what} needs {count} elements of {es} bytes, got "
                         f"{t.numel()} of {t.element_size()}")


def _check_fwd_io(fn, d, x=None, spk=None):
    rows = d.T * d.B
    _need(fn, x, d.in_dtype, rows * d.n_in, "x")
    if d.out_dtype == SPK_BITS:
        _need(fn, spk, U8, rows * d.n_out // 8, "spk_out (packed bits)")
    else:
        _need(fn, spk, d.out_dtype, rows * d.n_out, "spk_out")


def snn_layer_saved_bytes(desc: LayerDesc) -> int:
    return int(lib().snn_layer_saved_bytes(ctypes.byref(desc)))


def snn_layer_saved_layout(desc: LayerDesc) -> SavedLayout:
    out = SavedLayout()
    _check("snn_layer_saved_layout", lib().snn_layer_saved_layout(ctypes.byref(desc),
                                                                  ctypes.byref(out)))
    return out


def saved_parts(desc: LayerDesc, saved):
    """Views of a saved-state buffer (uint8 tensor of snn_layer_saved_bytes):
    (currents fp32 [T,B,n_out] or None, checkpoints fp32, pool selection u8
    [T,B,n_out] or None), at the offsets the library reports."""
    lay = snn_layer_saved_layout(desc)
    T, B, n = desc.T, desc.B, desc.n_out
    cur = None
    if lay.cur_bytes:
        cur = saved[lay.cur_offset: lay.cur_offset + T * B * n * 4].view(
            __import__("torch").float32).view(T, B, n)
    ck = saved[lay.ckpt_offset: lay.ckpt_offset + lay.ckpt_bytes].view(
        __import__("torch").float32)
    pool = None
    if lay.pool_bytes:
        pool = saved[lay.pool_offset: lay.pool_offset + T * B * n].view(T, B, n)
    return cur, ck, pool


def ckpt_buffer(desc: LayerDesc, device="cuda"):
    """A device buffer for the checkpoints of snn_neuron_fwd / snn_neuron_bwd."""
    import torch
    lay = snn_layer_saved_layout(desc)
    return torch.empty(max(64, lay.ckpt_bytes // 4), dtype=torch.float32, device=device)


def snn_layer_dcur_t_bytes(desc: LayerDesc) -> int:
    return int(lib().snn_layer_dcur_t_bytes(ctypes.byref(desc)))


def _dcur_t_written(desc: LayerDesc) -> int:
    """Bytes snn_neuron_bwd writes to a dcur_t argument: the layer's operand
    when its weight gradient takes one, else the transposed layout
    ([P][n_out][T*B] 16-bit, P = 3 for an fp32 dL/dI)."""
    n = snn_layer_dcur_t_bytes(desc)
    if n > 0:
        return n
    return (3 if desc.grad_dtype == F32 else 1) * desc.n_out * desc.T * desc.B * 2


def snn_layer_dcur_t_layout(desc: LayerDesc) -> int:
    """DCUR_T_TRANSPOSED or DCUR_T_PLANES: the layout of the dcur_t operand
    snn_neuron_bwd writes for this layer."""
    return int(lib().snn_layer_dcur_t_layout(ctypes.byref(desc)))


def snn_layer_workspace_bytes(desc: LayerDesc) -> int:
    return int(lib().snn_layer_workspace_bytes(ctypes.byref(desc)))


def snn_loss_workspace_bytes(kind: int, B: int, K: int) -> int:
    return int(lib().snn_loss_workspace_bytes(kind, B, K))


def snn_layer_fwd(desc, x, w, bias, v, spk_out, saved, counts, ws, stream=None):
    _check_fwd_io("snn_layer_fwd", desc, x, spk_out)
    _check("snn_layer_fwd", lib().snn_layer_fwd(
        ctypes.byref(desc), _p(x), _p(w), _p(bias), _p(v), _p(spk_out), _p(saved), _p(counts),
        _p(ws), _nbytes(ws), _stream(stream)))


def snn_layer_bwd(desc, grad_kind, g, x, w, v, saved, grad_w, grad_b, grad_v, grad_x, ws,
                  stream=None):
    _check_fwd_io("snn_layer_bwd", desc, x)
    gi = _grad_in(grad_kind, g)
    _check("snn_layer_bwd", lib().snn_layer_bwd(
        ctypes.byref(desc), ctypes.byref(gi), _p(x), _p(w), _p(v), _p(saved), _p(grad_w),
        _p(grad_b), _p(grad_v), _p(grad_x), _p(ws), _nbytes(ws), _stream(stream)))


def snn_loss(kind, B, K, P, counts, labels, targets, loss, grad_counts, ws, stream=None):
    _check("snn_loss", lib().snn_loss(kind, B, K, P, _p(counts), _p(labels), _p(targets),
                                      _p(loss), _p(grad_counts), _p(ws), _nbytes(ws),
                                      _stream(stream)))


def snn_loss_noalloc(kind, B, K, P, counts, labels, targets, loss, grad_counts, stream=None):
    _check("snn_loss_noalloc", lib().snn_loss_noalloc(kind, B, K, P, _p(counts), _p(labels),
                                                      _p(targets), _p(loss), _p(grad_counts),
                                                      _stream(stream)))


def fused_desc(hidden, readout, loss_kind, pop=1, wait_limit=0) -> FusedDesc:
    f = FusedDesc()
    f.hidden, f.readout = hidden, readout
    f.loss_kind, f.pop, f.wait_limit, f.reserved = loss_kind, pop, wait_limit, 0
    return f


def snn_fused_step_check(fd) -> int:
    return lib().snn_fused_step_check(ctypes.byref(fd))


def snn_fused_step_workspace_bytes(fd) -> int:
    return lib().snn_fused_step_workspace_bytes(ctypes.byref(fd))


def snn_fused_step(fd, x, w0, b0, w1, b1, labels, targets, loss, counts, gw0, gb0, gw1, gb1,
                   status, ws, stream=None, spk_hidden=None):
    h, r = fd.hidden, fd.readout
    _need("snn_fused_step", x, U8, h.T * h.B * h.n_in, "x")
    _need("snn_fused_step", w0, F32, h.n_out * h.n_in, "w0")
    _need("snn_fused_step", w1, F32, r.n_out * r.n_in, "w1")
    _need("snn_fused_step", gw0, F32, h.n_out * h.n_in, "grad_w0")
    _need("snn_fused_step", gw1, F32, r.n_out * r.n_in, "grad_w1")
    _need("snn_fused_step", counts, F32, h.B * r.n_out, "counts")
    _need("snn_fused_step", b0, F32, h.n_out, "b0")
    _need("snn_fused_step", b1, F32, r.n_out, "b1")
    _need("snn_fused_step", gb0, F32, h.n_out, "grad_b0")
    _need("snn_fused_step", gb1, F32, r.n_out, "grad_b1")
    _need("snn_fused_step", loss, F32, 1, "loss")
    _need("snn_fused_step", status, I32, 1, "status")
    _need("snn_fused_step", spk_hidden, U8, h.T * h.B * h.n_out, "spk_hidden")
    if fd.loss_kind == LOSS_CE_COUNT:
        _need("snn_fused_step", labels, I32, h.B, "labels")
    else:
        _need("snn_fused_step", targets, F32, h.B * (r.n_out // max(fd.pop, 1)), "targets")
    _check("snn_fused_step", lib().snn_fused_step(
        ctypes.byref(fd), _p(x), _p(w0), _p(b0), _p(w1), _p(b1), _p(labels), _p(targets),
        _p(loss), _p(counts), _p(spk_hidden), _p(gw0), _p(gb0), _p(gw1), _p(gb1), _p(status),
        _p(ws), _nbytes(ws), _stream(stream)))


def snn_synapse_fwd(desc, x, w, bias, cur, pool_arg, ws, stream=None):
    _check_fwd_io("snn_synapse_fwd", desc, x)
    _check("snn_synapse_fwd", lib().snn_synapse_fwd(
        ctypes.byref(desc), _p(x), _p(w), _p(bias), _p(cur), _p(pool_arg), _p(ws), _nbytes(ws),
        _stream(stream)))


def snn_neuron_fwd(desc, cur, v, spk_out, ckpt, counts, stream=None, u_out=None):
    """ckpt: checkpoints (ckpt_buffer); u_out: the membrane of every step, or None."""
    _check_fwd_io("snn_neuron_fwd", desc, None, spk_out)
    _need("snn_neuron_fwd", u_out, F32, desc.T * desc.B * desc.n_out, "u_out")
    _need("snn_neuron_fwd", ckpt, F32, snn_layer_saved_layout(desc).ckpt_bytes // 4, "ckpt")
    _check("snn_neuron_fwd", lib().snn_neuron_fwd(
        ctypes.byref(desc), _p(cur), _p(v), _p(spk_out), _p(ckpt), _p(u_out), _p(counts),
        _stream(stream)))


def snn_neuron_bwd(desc, grad_kind, g, v, cur, ckpt, dcur, grad_b, grad_v, ws, stream=None,
                   dcur_scale=None, dcur_t=None):
    """cur, ckpt: the forward's currents and checkpoints.  dcur_scale: device
    fp32 scalar receiving the power of two an fp16 dcur is scaled by
    (required for grad_dtype F16).  dcur_t: the weight gradient's operand in
    the layout snn_layer_dcur_t_layout names (transposed, or an fp32 dL/dI's
    three bf16 planes; snn_layer_dcur_t_bytes), or None; dcur may then be
    None."""
    if dcur_t is not None and dcur_t.numel() * dcur_t.element_size() < _dcur_t_written(desc):
        raise ValueError("snn_neuron_bwd: dcur_t smaller than the operand the scan writes")
    _need("snn_neuron_bwd", cur, F32, desc.T * desc.B * desc.n_out, "cur")
    _need("snn_neuron_bwd", ckpt, F32, snn_layer_saved_layout(desc).ckpt_bytes // 4, "ckpt")
    _need("snn_neuron_bwd", dcur, desc.grad_dtype if desc.synapse != SYN_NONE else F32,
          desc.T * desc.B * desc.n_out, "dcur")
    gi = _grad_in(grad_kind, g)
    _check("snn_neuron_bwd", lib().snn_neuron_bwd(
        ctypes.byref(desc), ctypes.byref(gi), _p(v), _p(cur), _p(ckpt), _p(dcur), _p(dcur_t),
        _p(dcur_scale), _p(grad_b), _p(grad_v), _p(ws), _nbytes(ws), _stream(stream)))


def snn_synapse_bwd(desc, dcur, pool_arg, x, w, grad_w, grad_x, ws, stream=None,
                    dcur_scale=None, dcur_t=None):
    _check_fwd_io("snn_synapse_bwd", desc, x)
    _need("snn_synapse_bwd", dcur, desc.grad_dtype, desc.T * desc.B * desc.n_out, "dcur")
    if dcur_t is not None and dcur_t.numel() * dcur_t.element_size() < \
            snn_layer_dcur_t_bytes(desc):
        raise ValueError("snn_synapse_bwd: dcur_t smaller than snn_layer_dcur_t_bytes")
    _check("snn_synapse_bwd", lib().snn_synapse_bwd(
        ctypes.byref(desc), _p(dcur), _p(dcur_t), _p(dcur_scale), _p(pool_arg), _p(x), _p(w),
        _p(grad_w), _p(grad_x), _p(ws), _nbytes(ws), _stream(stream)))


def snn_adamw(tensors, step, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2,
              stream=None):
    """tensors: sequence of (param, grad, m, v, param_half or None) device
    tensors (fp32, param_half fp16), all updated in one fused pass."""
    arr = (AdamwTensor * max(1, len(tensors)))()
    for i, (p, g, m, v, h) in enumerate(tensors):
        arr[i] = AdamwTensor(_p(p), _p(g), _p(m), _p(v), _p(h), p.numel())
    hp = AdamwHparams(lr, betas[0], betas[1], eps, weight_decay, step)
    _check("snn_adamw", lib().snn_adamw(arr, len(tensors), ctypes.byref(hp), _stream(stream)))


# --------------------------------------------------------------------------
# leaky sequence block
# --------------------------------------------------------------------------
def linattn_desc(q, k, v, o, scale=None, forward_only=False) -> LinattnDesc:
    """Descriptor of linear attention over q [T,B,heads,d_k], k [T,B,kv_heads,d_k],
    v [T,B,kv_heads,d_v] and o [T,B,heads,d_v]: tensors of one dtype, each row
    contiguous, strided over time, sequence and head (scale: 1/sqrt(d_k) if None;
    forward_only: for prompts and steps, whose workspace leaves out the backward's).
    Later calls may pass other tensors of the same shapes and strides."""
    T, B, H, DK = q.shape
    KV, DV = k.shape[2], v.shape[3]
    if k.shape != (T, B, KV, DK) or v.shape != (T, B, KV, DV) or o.shape != (T, B, H, DV):
        raise ValueError(f"linattn_desc: shapes {tuple(q.shape)}, {tuple(k.shape)}, "
                         f"{tuple(v.shape)}, {tuple(o.shape)} do not go together")
    if any(t.dtype != q.dtype for t in (k, v, o)):
        raise ValueError("linattn_desc: q, k, v and o must have one dtype")
    if any(t.stride(3) != 1 and t.shape[3] > 1 and t.numel() for t in (q, k, v, o)):
        raise ValueError("linattn_desc: each head's values must be contiguous")
    S = ctypes.c_int64 * 3
    return LinattnDesc(T, B, H, KV, DK, DV, _dtype_code(q), DK ** -0.5 if scale is None else scale,
                       *(S(*t.stride()[:3]) if t.numel() else S() for t in (q, k, v, o)),
                       int(forward_only))


def _need_heads(fn, what, t, dtype, shape, stride):
    """A strided argument of the shape, type and strides the descriptor has
    (dimensions of one element have any stride)."""
    if t is None or isinstance(t, int):
        return
    if t.dtype is dtype and t.shape == shape:
        st = t.stride()
        if st[3] == 1 and list(st[:3]) == stride[:]:
            return
        if not t.numel() or st[3] == 1 and all(n == 1 or a == b
                                               for n, a, b in zip(shape, st, stride)):
            return
    raise ValueError(f"{fn}: {what} {tuple(t.shape)} {t.dtype} with strides {t.stride()} is not "
                     "what the descriptor says")


_torch_dtypes = {}  # by code, once torch is there


def _torch_dtype(code):
    if not _torch_dtypes:
        import torch
        _torch_dtypes.update({F32: torch.float32, F16: torch.float16, BF16: torch.bfloat16,
                              I32: torch.int32})
    return _torch_dtypes.get(code, _torch_dtypes[BF16])


def _need_linattn(fn, d, q, k, v, o, decay, prefix=""):
    dt, T, B, H, KV, DK, DV = (_torch_dtype(d.dtype), d.T, d.B, d.heads, d.kv_heads, d.d_k,
                               d.d_v)
    _need_heads(fn, prefix + "q", q, dt, (T, B, H, DK), d.q_stride)
    _need_heads(fn, prefix + "k", k, dt, (T, B, KV, DK), d.k_stride)
    _need_heads(fn, prefix + "v", v, dt, (T, B, KV, DV), d.v_stride)
    _need_heads(fn, "o or its gradient", o, dt, (T, B, H, DV), d.o_stride)
    _need_array(fn, decay, F32, H, "decay")


def _need_array(fn, t, dtype_code, count, what):
    """_need for an argument that must also be contiguous and of the type itself."""
    if t is None or isinstance(t, int):
        return
    dt = _torch_dtype(F32 if dtype_code == F32 else I32)
    if t.dtype is not dt or t.numel() < count or not t.is_contiguous():
        raise ValueError(f"{fn}: {what} needs {count} contiguous elements of {dt}, got "
                         f"{t.numel()} of {t.dtype}")


def snn_linattn_workspace_bytes(desc: LinattnDesc) -> int:
    return int(lib().snn_linattn_workspace_bytes(ctypes.byref(desc)))


def snn_linattn_fwd(desc, q, k, v, decay, lens, state_in, o, state_out, ws, stream=None):
    """Whole sequences: o and, where given, the state after each (from state_in,
    or zeros).  lens: int32 [B] lengths, or None."""
    fn, S = "snn_linattn_fwd", desc.B * desc.heads * desc.d_k * desc.d_v
    _need_linattn(fn, desc, q, k, v, o, decay)
    _need_array(fn, lens, I32, desc.B, "lens")
    _need_array(fn, state_in, F32, S, "state_in")
    _need_array(fn, state_out, F32, S, "state_out")
    _check(fn, lib().snn_linattn_fwd(
        ctypes.byref(desc), _p(q), _p(k), _p(v), _p(decay), _p(lens), _p(state_in), _p(o),
        _p(state_out), _p(ws), _nbytes(ws), _stream(stream)))


def snn_linattn_bwd(desc, q, k, v, decay, lens, state_in, grad_o, grad_state_out, grad_q, grad_k,
                    grad_v, grad_state_in, ws, stream=None):
    fn, S = "snn_linattn_bwd", desc.B * desc.heads * desc.d_k * desc.d_v
    _need_linattn(fn, desc, q, k, v, grad_o, decay)
    _need_linattn(fn, desc, grad_q, grad_k, grad_v, None, None, "grad_")
    _need_array(fn, lens, I32, desc.B, "lens")
    _need_array(fn, state_in, F32, S, "state_in")
    _need_array(fn, grad_state_out, F32, S, "grad_state_out")
    _need_array(fn, grad_state_in, F32, S, "grad_state_in")
    _check(fn, lib().snn_linattn_bwd(
        ctypes.byref(desc), _p(q), _p(k), _p(v), _p(decay), _p(lens), _p(state_in), _p(grad_o),
        _p(grad_state_out), _p(grad_q), _p(grad_k), _p(grad_v), _p(grad_state_in), _p(ws),
        _nbytes(ws), _stream(stream)))


def snn_linattn_step(desc, q, k, v, decay, slots, state_in, state_out, o, stream=None):
    """One token of every request; states [n_slots, heads, d_k, d_v] in pools
    (one and the same for an update in place), slots int32 [B] or None."""
    fn, n_slots = "snn_linattn_step", state_in.shape[0]
    S = n_slots * desc.heads * desc.d_k * desc.d_v
    _need_linattn(fn, desc, q, k, v, o, decay)
    _need_array(fn, slots, I32, desc.B, "slots")
    _need_array(fn, state_in, F32, S, "state_in")
    _need_array(fn, state_out, F32, S, "state_out")
    _check(fn, lib().snn_linattn_step(
        ctypes.byref(desc), _p(q), _p(k), _p(v), _p(decay), _p(slots), n_slots, _p(state_in),
        _p(state_out), _p(o), _stream(stream)))


_GATE = {"none": GATE_NONE, "mul": GATE_MUL, "sigmoid": GATE_SIGMOID, "silu": GATE_SILU}


def _row_stride(t):
    """Row stride of a tensor [..., n] whose leading dimensions are one row index
    and whose rows are contiguous (ValueError for others)."""
    n, st = t.shape, t.stride()
    if t.numel() == 0:
        return max(n[-1], 1)
    if n[-1] > 1 and st[-1] != 1:
        raise ValueError("row tensors must be contiguous within a row")
    ld, rows = None, 1
    for size, s in zip(n[-2::-1], st[-2::-1]):
        if size == 1:
            continue
        if ld is None:
            ld = s
        elif s != ld * rows:
            raise ValueError(f"rows of a tensor of shape {tuple(n)} and strides {st} have no "
                             "single stride")
        rows *= size
    return max(n[-1], 1) if ld is None else ld


def gate_norm_desc(x, y=None, gate=None, groups=1, act="none", eps=1e-6, h=None,
                   ckpt_block=128) -> GateNormDesc:
    """Descriptor of the norms around a block: x [..., n] the residual stream, y
    the block's output and gate (or None), with act "none", "mul", "sigmoid" or
    "silu"; y's norm is taken over each of `groups` parts of a row.  Later calls
    may pass other tensors of the same strides; x_out has x's, h those of the h
    given here (contiguous rows of y's dtype, or x's without y, if None).  ckpt_block:
    values that share a scale in 8-bit checkpoints of y and the gate; a block
    should lie within one group."""
    n = x.shape[-1]
    rows = x.numel() // n if n else 0
    for t in (y, gate, h):
        if t is not None and t.shape != x.shape:
            raise ValueError(f"gate_norm_desc: shapes {tuple(x.shape)} and {tuple(t.shape)}")
    yt = _dtype_code(y if y is not None else h if h is not None else x)
    return GateNormDesc(rows, n, groups, _GATE[act], _dtype_code(x), yt, eps, ckpt_block,
                        _row_stride(x),
                        n if y is None else _row_stride(y),
                        n if gate is None else _row_stride(gate),
                        n if h is None else _row_stride(h))


def _need_rows(fn, what, t, d, dtype, ld):
    if t is None or isinstance(t, int):
        return
    n, rows, shape = d.n, d.rows, t.shape
    if t.dtype is dtype and shape[-1] == n and t.numel() == rows * n:
        if len(shape) == 2 and t.stride() == (ld, 1):
            return
        # a single row may have any stride, its values must lie together all the same
        if _row_stride(t) == ld or rows <= 1:
            return
    raise ValueError(f"{fn}: {what} {tuple(t.shape)} {t.dtype} with strides {t.stride()} is not "
                     "what the descriptor says")


def _need_ckpt(fn, what, t, rows, n, block):
    if t is None or isinstance(t, int):
        return
    need = snn_checkpoint_bytes(rows, n, block)
    if not t.is_contiguous() or _nbytes(t) < need:
        raise ValueError(f"{fn}: {what} needs {need} contiguous bytes")


def snn_gate_norm_workspace_bytes(desc: GateNormDesc) -> int:
    return int(lib().snn_gate_norm_workspace_bytes(ctypes.byref(desc)))


def snn_gate_norm_fwd(desc, x, y, gate, w_post, scale, w_pre, x_out, h, y_ckpt=None,
                      gate_ckpt=None, stream=None):
    """x_out = x + scale norm(y) w_post act(gate) and h = norm(x_out) w_pre (y
    None: h = norm(x) w_pre alone), with y and the gate stored in 8 bits where
    y_ckpt and gate_ckpt are given."""
    fn, d = "snn_gate_norm_fwd", desc
    xt, yt, n = _torch_dtype(d.x_dtype), _torch_dtype(d.y_dtype), d.n
    _need_rows(fn, "x", x, d, xt, d.ld_x)
    _need_rows(fn, "x_out", x_out, d, xt, d.ld_x)
    _need_rows(fn, "y", y, d, yt, d.ld_y)
    _need_rows(fn, "gate", gate, d, yt, d.ld_g)
    _need_rows(fn, "h", h, d, yt, d.ld_h)
    _need_array(fn, w_post, F32, n, "w_post")
    _need_array(fn, scale, F32, n, "scale")
    _need_array(fn, w_pre, F32, n, "w_pre")
    _need_ckpt(fn, "y_ckpt", y_ckpt, d.rows, n, d.ckpt_block)
    _need_ckpt(fn, "gate_ckpt", gate_ckpt, d.rows, n, d.ckpt_block)
    _check(fn, lib().snn_gate_norm_fwd(
        ctypes.byref(d), _p(x), _p(y), _p(gate), _p(w_post), _p(scale), _p(w_pre), _p(x_out),
        _p(h), _p(y_ckpt), _p(gate_ckpt), _stream(stream)))


def snn_gate_norm_bwd(desc, grad_x_out, grad_h, x_out, y, gate, y_ckpt, gate_ckpt, w_post, scale,
                      w_pre, grad_x, grad_y, grad_gate, grad_w_post, grad_scale, grad_w_pre, ws,
                      stream=None):
    """The backward of snn_gate_norm_fwd, from y and gate or from their 8-bit
    checkpoints."""
    fn, d = "snn_gate_norm_bwd", desc
    xt, yt = _torch_dtype(d.x_dtype), _torch_dtype(d.y_dtype)
    for what, t in (("grad_x_out", grad_x_out), ("x_out", x_out), ("grad_x", grad_x)):
        _need_rows(fn, what, t, d, xt, d.ld_x)
    for what, t, ld in (("y", y, d.ld_y), ("grad_y", grad_y, d.ld_y), ("gate", gate, d.ld_g),
                        ("grad_gate", grad_gate, d.ld_g), ("grad_h", grad_h, d.ld_h)):
        _need_rows(fn, what, t, d, yt, ld)
    for what, t in (("w_post", w_post), ("scale", scale), ("w_pre", w_pre),
                    ("grad_w_post", grad_w_post), ("grad_scale", grad_scale),
                    ("grad_w_pre", grad_w_pre)):
        _need_array(fn, t, F32, d.n, what)
    for what, t in (("y_ckpt", y_ckpt), ("gate_ckpt", gate_ckpt)):
        _need_ckpt(fn, what, t, d.rows, d.n, d.ckpt_block)
    _check(fn, lib().snn_gate_norm_bwd(
        ctypes.byref(d), _p(grad_x_out), _p(grad_h), _p(x_out), _p(y), _p(gate), _p(y_ckpt),
        _p(gate_ckpt), _p(w_post), _p(scale), _p(w_pre), _p(grad_x), _p(grad_y), _p(grad_gate),
        _p(grad_w_post), _p(grad_scale), _p(grad_w_pre), _p(ws), _nbytes(ws), _stream(stream)))


def snn_checkpoint_bytes(rows: int, n: int, block: int = 128) -> int:
    return int(lib().snn_checkpoint_bytes(rows, n, block))


def _checkpoint(fn, x, ckpt, block, args, stream):
    n = x.shape[-1]
    rows = x.numel() // n if n else 0
    _need_ckpt(fn, "ckpt", ckpt, rows, n, block)
    _check(fn, getattr(lib(), fn)(rows, n, block, _row_stride(x), _dtype_code(x), *args,
                                  _stream(stream)))


def snn_checkpoint_save(x, ckpt, block=128, stream=None):
    """Stores x [..., n] in 8 bits in ckpt (snn_checkpoint_bytes(rows, n, block)
    bytes), `block` values to a scale."""
    _checkpoint("snn_checkpoint_save", x, ckpt, block, (_p(x), _p(ckpt)), stream)


def snn_checkpoint_load(ckpt, x, block=128, stream=None):
    """Reads the checkpoint of x's shape back into x (any of its dtypes)."""
    _checkpoint("snn_checkpoint_load", x, ckpt, block, (_p(ckpt), _p(x)), stream)


# --------------------------------------------------------------------------
# selective leaky block
# --------------------------------------------------------------------------
def _fit(fn, *sizes):
    """A descriptor's sizes: a field of 32 bits would keep the rest of a larger one."""
    if any(not 0 <= n < 1 << 31 for n in sizes):
        raise ValueError(f"{fn}: sizes {sizes} do not fit 32 bits")
    return sizes


def _strides(fn, t, dims):
    """Strides of the leading `dims` dimensions of a tensor whose last is contiguous
    (0 for a dimension of one element: it has none to speak of)."""
    if t.numel() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{fn}: a row's values must be contiguous")
    st = [s if n > 1 and t.numel() else 0 for n, s in zip(t.shape[:dims], t.stride())]
    return (ctypes.c_int64 * dims)(*st)


def _seen(desc, **tensors):
    """Keeps with a descriptor the layouts it was made from: the usual arguments' check is
    then a comparison or three (a small call is bound by the host)."""
    desc.layouts = {k: (t.dtype, t.shape, t.stride()) for k, t in tensors.items()
                    if t is not None}
    desc.fields = bytes(desc)
    return desc


def _layouts(desc):
    """What _seen kept, unless a field was changed since."""
    try:
        return desc.layouts if desc.fields == bytes(desc) else {}
    except AttributeError:  # a descriptor made by hand
        return {}


def _need_strided(fn, what, t, code, seen, shape, stride):
    """A strided argument of the shape, type and strides the descriptor has."""
    if t is None or isinstance(t, int):
        return
    if seen is not None and t.dtype is seen[0] and t.shape == seen[1] and t.stride() == seen[2]:
        return
    if t.dtype is _torch_dtype(code) and t.shape == shape:
        st = t.stride()
        if not t.numel() or (st[-1] == 1 or shape[-1] == 1) and all(
                n == 1 or a == b for n, a, b in zip(shape, st, stride)):
            return
    raise ValueError(f"{fn}: {what} {tuple(t.shape)} {t.dtype} with strides {t.stride()} is not "
                     "what the descriptor says")


def selscan_desc(u, dt, b, c, y, z=None, delta_softplus=True, forward_only=False) -> SelscanDesc:
    """Descriptor of a selective scan over u, dt, y and the gate z (or None) [T,B,n],
    b and c [T,B,groups,states]: tensors of one dtype, each row contiguous, strided over
    time, sequence and group (forward_only: for prompts and steps, for which nothing is
    saved).  Later calls may pass other tensors of the same shapes and strides."""
    fn = "selscan_desc"
    T, B, n = u.shape
    if any(t is not None and t.shape != u.shape for t in (dt, y, z)) or b.dim() != 4 or \
            b.shape[:2] != (T, B) or c.shape != b.shape:
        raise ValueError(f"{fn}: shapes {[tuple(t.shape) for t in (u, dt, b, c, y)]} do not go "
                         "together")
    if any(t is not None and t.dtype != u.dtype for t in (dt, b, c, y, z)):
        raise ValueError(f"{fn}: u, dt, b, c, y and z must have one dtype")
    d = SelscanDesc(*_fit(fn, T, B, n, b.shape[3], b.shape[2]), _dtype_code(u),
                    int(delta_softplus), int(forward_only), *(_strides(fn, t, 2) for t in (u, dt)),
                    _strides(fn, z if z is not None else u, 2), _strides(fn, y, 2),
                    _strides(fn, b, 3), _strides(fn, c, 3))
    return _seen(d, u=u, dt=dt, z=z, y=y, b=b, c=c)


def snn_selscan_saved_bytes(desc: SelscanDesc) -> int:
    return int(lib().snn_selscan_saved_bytes(ctypes.byref(desc)))


def snn_selscan_workspace_bytes(desc: SelscanDesc) -> int:
    return int(lib().snn_selscan_workspace_bytes(ctypes.byref(desc)))


def _need_selscan(fn, d, u, dt, a, b, c, skip, dt_bias, z, y, prefix=""):
    n, code, seen = d.n, d.dtype, _layouts(d).get
    rows, vecs = (d.T, d.B, n), (d.T, d.B, d.groups, d.states)
    _need_strided(fn, prefix + "u", u, code, seen("u"), rows, d.u_stride)
    _need_strided(fn, prefix + "dt", dt, code, seen("dt"), rows, d.dt_stride)
    _need_strided(fn, prefix + "z", z, code, seen("z"), rows, d.z_stride)
    _need_strided(fn, "y or its gradient", y, code, seen("y"), rows, d.y_stride)
    _need_strided(fn, prefix + "b", b, code, seen("b"), vecs, d.b_stride)
    _need_strided(fn, prefix + "c", c, code, seen("c"), vecs, d.c_stride)
    _need_array(fn, a, F32, d.states * n, prefix + "a")
    _need_array(fn, skip, F32, n, prefix + "skip")
    _need_array(fn, dt_bias, F32, n, prefix + "dt_bias")


def _need_bytes(fn, t, need, what):
    if t is None or isinstance(t, int):
        return
    if not t.is_contiguous() or _nbytes(t) < need:
        raise ValueError(f"{fn}: {what} needs {need} contiguous bytes")


def snn_selscan_fwd(desc, u, dt, a, b, c, skip, dt_bias, z, lens, state_in, y, state_out, saved,
                    ws, stream=None):
    """Whole sequences: y and, where given, the states after each (from state_in, or
    zeros); saved (snn_selscan_saved_bytes) is for the backward.  lens: int32 [B] lengths,
    or None."""
    fn, d = "snn_selscan_fwd", desc
    _need_selscan(fn, d, u, dt, a, b, c, skip, dt_bias, z, y)
    _need_array(fn, lens, I32, d.B, "lens")
    for what, t in (("state_in", state_in), ("state_out", state_out)):
        _need_array(fn, t, F32, d.B * d.states * d.n, what)
    if saved is not None:
        _need_bytes(fn, saved, snn_selscan_saved_bytes(d), "saved")
    _check(fn, lib().snn_selscan_fwd(
        ctypes.byref(d), _p(u), _p(dt), _p(a), _p(b), _p(c), _p(skip), _p(dt_bias), _p(z),
        _p(lens), _p(state_in), _p(y), _p(state_out), _p(saved), _p(ws), _nbytes(ws),
        _stream(stream)))


def snn_selscan_bwd(desc, u, dt, a, b, c, skip, dt_bias, z, lens, saved, grad_y, grad_state_out,
                    grad_u, grad_dt, grad_a, grad_b, grad_c, grad_skip, grad_dt_bias, grad_z,
                    grad_state_in, ws, stream=None):
    fn, d = "snn_selscan_bwd", desc
    _need_selscan(fn, d, u, dt, a, b, c, skip, dt_bias, z, grad_y)
    _need_selscan(fn, d, grad_u, grad_dt, grad_a, grad_b, grad_c, grad_skip, grad_dt_bias, grad_z,
                  None, "grad_")
    _need_array(fn, lens, I32, d.B, "lens")
    for what, t in (("grad_state_out", grad_state_out), ("grad_state_in", grad_state_in)):
        _need_array(fn, t, F32, d.B * d.states * d.n, what)
    _need_bytes(fn, saved, snn_selscan_saved_bytes(d), "saved")
    _check(fn, lib().snn_selscan_bwd(
        ctypes.byref(d), _p(u), _p(dt), _p(a), _p(b), _p(c), _p(skip), _p(dt_bias), _p(z),
        _p(lens), _p(saved), _p(grad_y), _p(grad_state_out), _p(grad_u), _p(grad_dt), _p(grad_a),
        _p(grad_b), _p(grad_c), _p(grad_skip), _p(grad_dt_bias), _p(grad_z), _p(grad_state_in),
        _p(ws), _nbytes(ws), _stream(stream)))


def snn_selscan_step(desc, u, dt, a, b, c, skip, dt_bias, z, slots, state_in, state_out, y,
                     stream=None):
    """One token of every request; states [n_slots, states, n] in pools (one and the same
    for an update in place), slots int32 [B] or None."""
    fn, d, n_slots = "snn_selscan_step", desc, state_in.shape[0]
    _need_selscan(fn, d, u, dt, a, b, c, skip, dt_bias, z, y)
    _need_array(fn, slots, I32, d.B, "slots")
    for what, t in (("state_in", state_in), ("state_out", state_out)):
        _need_array(fn, t, F32, n_slots * d.states * d.n, what)
    _check(fn, lib().snn_selscan_step(
        ctypes.byref(d), _p(u), _p(dt), _p(a), _p(b), _p(c), _p(skip), _p(dt_bias), _p(z),
        _p(slots), n_slots, _p(state_in), _p(state_out), _p(y), _stream(stream)))


def shortconv_desc(x, y, width, act="none") -> ShortconvDesc:
    """Descriptor of the short causal convolution of x into y [T,B,n], each row contiguous,
    strided over time and sequence, with `width` taps and act "none" or "silu".  Later
    calls may pass other tensors of the same shapes and strides."""
    fn = "shortconv_desc"
    if x.dim() != 3 or x.shape != y.shape or x.dtype != y.dtype:
        raise ValueError(f"{fn}: {tuple(x.shape)} {x.dtype} and {tuple(y.shape)} {y.dtype} do "
                         "not go together")
    d = ShortconvDesc(*_fit(fn, *x.shape, width), _GATE[act], _dtype_code(x), _strides(fn, x, 2),
                      _strides(fn, y, 2))
    return _seen(d, x=x, y=y)


def snn_shortconv_workspace_bytes(desc: ShortconvDesc) -> int:
    return int(lib().snn_shortconv_workspace_bytes(ctypes.byref(desc)))


def _need_shortconv(fn, d, x, w, bias, y, prefix=""):
    rows, code, seen = (d.T, d.B, d.n), d.dtype, _layouts(d).get
    _need_strided(fn, prefix + "x", x, code, seen("x"), rows, d.x_stride)
    _need_strided(fn, "y or its gradient", y, code, seen("y"), rows, d.y_stride)
    _need_array(fn, w, F32, d.width * d.n, prefix + "w")
    _need_array(fn, bias, F32, d.n, prefix + "bias")


def snn_shortconv_fwd(desc, x, w, bias, lens, state_in, y, state_out, stream=None):
    """Whole sequences: y and, where given, the last width - 1 inputs (after those of
    state_in, or zeros), fp32 [B, width - 1, n].  lens: int32 [B] lengths, or None."""
    fn, d = "snn_shortconv_fwd", desc
    _need_shortconv(fn, d, x, w, bias, y)
    _need_array(fn, lens, I32, d.B, "lens")
    for what, t in (("state_in", state_in), ("state_out", state_out)):
        _need_array(fn, t, F32, d.B * (d.width - 1) * d.n, what)
    _check(fn, lib().snn_shortconv_fwd(
        ctypes.byref(d), _p(x), _p(w), _p(bias), _p(lens), _p(state_in), _p(y), _p(state_out),
        _stream(stream)))


def snn_shortconv_bwd(desc, x, w, bias, lens, state_in, grad_y, grad_state_out, grad_x, grad_w,
                      grad_bias, grad_state_in, ws, stream=None):
    fn, d = "snn_shortconv_bwd", desc
    _need_shortconv(fn, d, x, w, bias, grad_y)
    _need_shortconv(fn, d, grad_x, grad_w, grad_bias, None, "grad_")
    _need_array(fn, lens, I32, d.B, "lens")
    for what, t in (("state_in", state_in), ("grad_state_out", grad_state_out),
                    ("grad_state_in", grad_state_in)):
        _need_array(fn, t, F32, d.B * (d.width - 1) * d.n, what)
    _check(fn, lib().snn_shortconv_bwd(
        ctypes.byref(d), _p(x), _p(w), _p(bias), _p(lens), _p(state_in), _p(grad_y),
        _p(grad_state_out), _p(grad_x), _p(grad_w), _p(grad_bias), _p(grad_state_in), _p(ws),
        _nbytes(ws), _stream(stream)))


def snn_shortconv_step(desc, x, w, bias, slots, state_in, state_out, y, stream=None):
    """One token of every request; the last inputs [n_slots, width - 1, n] in pools (one
    and the same for an update in place), slots int32 [B] or None."""
    fn, d, n_slots = "snn_shortconv_step", desc, state_in.shape[0]
    _need_shortconv(fn, d, x, w, bias, y)
    _need_array(fn, slots, I32, d.B, "slots")
    for what, t in (("state_in", state_in), ("state_out", state_out)):
        _need_array(fn, t, F32, n_slots * (d.width - 1) * d.n, what)
    _check(fn, lib().snn_shortconv_step(
        ctypes.byref(d), _p(x), _p(w), _p(bias), _p(slots), n_slots, _p(state_in),
        _p(state_out), _p(y), _stream(stream)))


def layer_norm_desc(x, y=None, eps=1e-5) -> LayerNormDesc:
    """Descriptor of a layer norm of the rows of x [..., n] into y (contiguous rows of x's
    dtype if None).  Later calls may pass other tensors of the same strides."""
    n = x.shape[-1]
    if y is not None and y.shape != x.shape:
        raise ValueError(f"layer_norm_desc: shapes {tuple(x.shape)} and {tuple(y.shape)}")
    d = LayerNormDesc(*_fit("layer_norm_desc", x.numel() // n if n else 0, n), _dtype_code(x),
                      _dtype_code(x if y is None else y), eps, _row_stride(x),
                      n if y is None else _row_stride(y))
    return _seen(d, x=x, y=y)


def _need_norm_rows(fn, what, t, d, seen, code, ld):
    """_need_rows, first by the layout kept with the descriptor."""
    if t is None or seen is not None and t.__class__ is not int and t.dtype is seen[0] and \
            t.shape == seen[1] and t.stride() == seen[2]:
        return
    _need_rows(fn, what, t, d, _torch_dtype(code), ld)


def snn_layer_norm_workspace_bytes(desc: LayerNormDesc) -> int:
    return int(lib().snn_layer_norm_workspace_bytes(ctypes.byref(desc)))


def snn_layer_norm_fwd(desc, x, w, b, y, stream=None):
    """y = (x - mean) / sqrt(var + eps) w + b over each row (w, b: None for ones, zeros)."""
    fn, d = "snn_layer_norm_fwd", desc
    n, seen = d.n, _layouts(d).get
    _need_norm_rows(fn, "x", x, d, seen("x"), d.x_dtype, d.ld_x)
    _need_norm_rows(fn, "y", y, d, seen("y"), d.y_dtype, d.ld_y)
    _need_array(fn, w, F32, n, "w")
    _need_array(fn, b, F32, n, "b")
    _check(fn, lib().snn_layer_norm_fwd(ctypes.byref(d), _p(x), _p(w), _p(b), _p(y),
                                        _stream(stream)))


def snn_layer_norm_bwd(desc, x, grad_y, grad_res, w, grad_x, grad_w, grad_b, ws, stream=None):
    """grad_x = grad_res (or None) + the norm's gradient; grad_w, grad_b sums over rows."""
    fn, d = "snn_layer_norm_bwd", desc
    seen = _layouts(d).get
    for what, t in (("x", x), ("grad_res", grad_res), ("grad_x", grad_x)):
        _need_norm_rows(fn, what, t, d, seen("x"), d.x_dtype, d.ld_x)
    _need_norm_rows(fn, "grad_y", grad_y, d, seen("y"), d.y_dtype, d.ld_y)
    for what, t in (("w", w), ("grad_w", grad_w), ("grad_b", grad_b)):
        _need_array(fn, t, F32, d.n, what)
    _check(fn, lib().snn_layer_norm_bwd(
        ctypes.byref(d), _p(x), _p(grad_y), _p(grad_res), _p(w), _p(grad_x), _p(grad_w),
        _p(grad_b), _p(ws), _nbytes(ws), _stream(stream)))


# --------------------------------------------------------------------------
# descriptors from plain layer specs
# --------------------------------------------------------------------------
_NEURON = {"leaky": LEAKY, "synaptic": SYNAPTIC, "rleaky": RLEAKY}


def layer_desc(spec: dict, T: int, B: int, in_dtype=U8, w_dtype=F32, out_dtype=U8,
               grad_dtype=F32, slope=25.0, reset_grad=RESET_DETACHED, flags=0) -> LayerDesc:
    d = LayerDesc()
    d.flags = flags
    d.T, d.B = T, B
    d.neuron = _NEURON[spec["neuron"]]
    d.beta = spec["beta"]
    d.alpha = spec.get("alpha", 0.0)
    d.threshold = spec.get("thr", 1.0)
    d.slope = slope
    d.reset_grad = reset_grad
    d.in_dtype, d.w_dtype, d.out_dtype, d.grad_dtype = in_dtype, w_dtype, out_dtype, grad_dtype
    if spec["kind"] == "dense":
        d.synapse = SYN_DENSE
        d.n_in, d.n_out = spec["n_in"], spec["n_out"]
    elif spec["kind"] == "conv":
        d.synapse = SYN_CONV5_POOL2
        d.c_in, d.h_in, d.w_in, d.c_out = spec["c_in"], spec["h"], spec["w"], spec["c_out"]
        d.n_in = d.c_in * d.h_in * d.w_in
        d.n_out = d.c_out * ((d.h_in - 4) // 2) * ((d.w_in - 4) // 2)
    else:
        d.synapse = SYN_NONE
        d.n_in = d.n_out = spec["n"]
        d.in_dtype = F32
    return d


class Network:
    """Device buffers and the layer-call sequence of one training step.

    All buffers are allocated once here (torch, device memory only); ``step``
    then only enqueues library calls on the current stream."""

    def __init__(self, wl, params, device="cuda", reset_grad=RESET_DETACHED, flags=0, fold=True,
                 spike_bits=False, input_bf16=False):
        import torch
        self.torch = torch
        self.wl = wl
        self.device = device
        T, B = wl.T, wl.B
        half = wl.dtype == "f16"
        self.descs = []
        self.W, self.b, self.v = [], [], []
        for li, spec in enumerate(wl.layers):
            in_dt = F32 if spec["kind"] == "none" else U8
            # input_bf16: an fp32 net's input spikes given as bf16 0/1, the
            # operand type of its three-plane contractions (no widening pass
            # before the first layer's forward and weight gradient)
            if li == 0 and input_bf16 and not half and spec["kind"] == "dense":
                in_dt = BF16
            # half-precision nets hand dL/dI to the contractions in bf16, which
            # keeps fp32's exponent range for the small BPTT gradients
            d = layer_desc(spec, T, B, in_dtype=in_dt, w_dtype=F16 if half else F32,
                           out_dtype=U8, grad_dtype=BF16 if half else F32, slope=wl.slope,
                           reset_grad=reset_grad, flags=flags)
            self.descs.append(d)
            W, b = params[li][0], params[li][1]
            # recurrent weights of an 'rleaky' layer: (W, b, v)
            v = params[li][2] if len(params[li]) > 2 else None
            self.v.append(None if v is None else torch.as_tensor(np.ascontiguousarray(
                v, np.float32)).to(device))
            if W is None:
                self.W.append(None)
                self.b.append(None)
            else:
                wdt = torch.float16 if half else torch.float32
                self.W.append(torch.as_tensor(np.ascontiguousarray(W)).to(device=device, dtype=wdt))
                self.b.append(torch.as_tensor(np.ascontiguousarray(b)).to(device=device,
                                                                         dtype=torch.float32))
        u8 = torch.uint8
        # Spikes that feed a large fp16 contraction (a dense layer above with
        # at least 256 outputs) are written as fp16 0/1 by the scan, the
        # operand type that contraction stages directly; other spikes as bytes.
        for li in range(len(self.descs) - 1):
            up = self.descs[li + 1]
            if half and up.synapse == SYN_DENSE and up.n_out >= 256 and up.n_in >= 256:
                self.descs[li].out_dtype = F16
                up.in_dtype = F16
        # spike_bits: the last layer's spikes, which no contraction reads,
        # packed 64 to a word (layers of a multiple of 64 neurons)
        if spike_bits and self.descs[-1].n_out % 64 == 0:
            self.descs[-1].out_dtype = SPK_BITS
        self.spk = [torch.empty((T, B, d.n_out // 8 if d.out_dtype == SPK_BITS else d.n_out),
                                dtype=torch.float16 if d.out_dtype == F16 else u8, device=device)
                    for d in self.descs]
        self.in_shape = (T, B) + tuple(wl.in_shape)
        self.saved = [torch.empty(snn_layer_saved_bytes(d), dtype=u8, device=device)
                      for d in self.descs]
        # (currents, checkpoints, pool selection) views of each saved buffer
        self.layouts = [snn_layer_saved_layout(d) for d in self.descs]
        self.parts = [saved_parts(d, sv) for d, sv in zip(self.descs, self.saved)]
        self.gW = [None if w is None else torch.empty(w.shape, dtype=torch.float32, device=device)
                   for w in self.W]
        self.gb = [None if b is None else torch.empty(b.shape, dtype=torch.float32, device=device)
                   for b in self.b]
        self.gv = [None if v is None else torch.empty(v.shape, dtype=torch.float32, device=device)
                   for v in self.v]
        # dL/dx of layer l is the upstream gradient of layer l-1
        self.gx = [None] + [torch.empty((T, B, d.n_in), dtype=torch.float32, device=device)
                            for d in self.descs[1:]]
        if self.descs[0].synapse == SYN_NONE:
            self.gx[0] = torch.empty((T, B, self.descs[0].n_in), dtype=torch.float32, device=device)
        # A dense layer with at most 16 outputs (the readout) above a layer of
        # at least 64 neurons: its input gradient dx = dI W is folded into the
        # reverse scan of the layer below (SNN_GRAD_FOLD), which then reads the
        # readout's dL/dI (kept in dup) instead of a [T,B,n] gradient.
        n = len(self.descs)
        self.fold = [fold and li + 1 < n and self.descs[li + 1].synapse == SYN_DENSE
                     and self.descs[li + 1].n_out <= 16 and self.descs[li].n_out >= 64
                     for li in range(n)]
        gdt = {F32: torch.float32, BF16: torch.bfloat16, F16: torch.float16}
        self.dup = [None] * n
        for li in range(n - 1):
            if self.fold[li]:
                self.gx[li + 1] = None
        # The fp16 net's gradient operand dL/dI: fp16 scaled by a power of two
        # (one MFMA pass against the fp16 weights of the input gradient) for
        # layers whose input gradient is a contraction; bf16 otherwise (the
        # weight gradient against spikes is one pass in either type).  The
        # scale needs a bound of the upstream gradient: cheap for a broadcast
        # or folded one, one extra read of a full [T,B,n] gradient otherwise.
        self.scale = [None] * n
        for li, d in enumerate(self.descs):
            if not half or d.synapse != SYN_DENSE or d.neuron == RLEAKY:
                continue
            if li > 0 and self.gx[li] is not None:
                d.grad_dtype = F16
                self.scale[li] = torch.empty(4, dtype=torch.float32, device=device)
        for li in range(n - 1):
            if self.fold[li]:
                up = self.descs[li + 1]
                self.dup[li + 1] = torch.empty((T, B, up.n_out), dtype=gdt[up.grad_dtype],
                                               device=device)
        # K classes, P output neurons per class (a population code when P > 1)
        self.P = getattr(wl, "pop", 1)
        n_last = self.descs[-1].n_out
        assert n_last % self.P == 0, (n_last, self.P)
        K = n_last // self.P
        self.K = K
        self.counts = torch.empty((B, n_last), dtype=torch.float32, device=device)
        self.loss = torch.empty(4, dtype=torch.float32, device=device)  # [0] is the loss
        self.gcounts = torch.empty((B, n_last), dtype=torch.float32, device=device)
        self.loss_kind = LOSS_CE_COUNT if wl.loss == "ce" else LOSS_MSE_COUNT
        ws = max([snn_layer_workspace_bytes(d) for d in self.descs] +
                 [snn_loss_workspace_bytes(self.loss_kind, B, K), 256])
        self.ws = torch.empty(ws, dtype=u8, device=device)
        # the reverse scan's transposed dL/dI for the weight gradient (stage
        # calls; the layer calls keep it in the workspace)
        self.dcur_t_bytes = [snn_layer_dcur_t_bytes(d) for d in self.descs]
        self.dcur_t_layout = [snn_layer_dcur_t_layout(d) for d in self.descs]
        self.transposed_operand = False
        self.dcur_t = torch.empty(max(self.dcur_t_bytes + [256]), dtype=u8, device=device)
        # The whole step as one cooperative launch (step_fused): two dense
        # layers on spike input with fp32 weights, small enough for one
        # co-resident grid; None where snn_fused_step_check refuses the net.
        self.fdesc = None
        if n == 2 and not half and all(d.synapse == SYN_DENSE for d in self.descs):
            fd = fused_desc(self.descs[0].copy(), self.descs[1].copy(), self.loss_kind, self.P)
            if snn_fused_step_check(fd) == 0:
                self.fdesc = fd
                self.fws = torch.empty(max(256, snn_fused_step_workspace_bytes(fd)), dtype=u8,
                                       device=device)
                self.fstatus = torch.zeros(4, dtype=torch.int32, device=device)

    def forward(self, x, stream=None):
        h = x
        n = len(self.descs)
        for li, d in enumerate(self.descs):
            snn_layer_fwd(d, h, self.W[li], self.b[li], self.v[li], self.spk[li], self.saved[li],
                          self.counts if li == n - 1 else None, self.ws, stream)
            h = self.spk[li]

    def loss_and_grad(self, labels=None, targets=None, stream=None):
        snn_loss(self.loss_kind, self.wl.B, self.K, self.P, self.counts, labels, targets,
                 self.loss, self.gcounts, self.ws, stream)

    def _grad_below(self, li):
        """The upstream gradient argument of layer li - 1."""
        if self.fold[li - 1]:
            return GRAD_FOLD, (self.dup[li], self.W[li])
        return GRAD_FULL, self.gx[li]

    def backward(self, x, stream=None):
        n = len(self.descs)
        kind, g = GRAD_BCAST, self.gcounts
        for li in range(n - 1, -1, -1):
            d = self.descs[li]
            xin = x if li == 0 else self.spk[li - 1]
            if self.dup[li] is not None:
                # dL/dI kept for the layer below; no dx of its own
                cur, ck, _ = self.parts[li]
                snn_neuron_bwd(d, kind, g, self.v[li], xin if cur is None else cur, ck,
                               self.dup[li], self.gb[li], self.gv[li], self.ws, stream,
                               dcur_scale=self.scale[li])
                snn_synapse_bwd(d, self.dup[li], self.pool_arg(li), xin, self.W[li], self.gW[li],
                                None, self.ws, stream, dcur_scale=self.scale[li])
            else:
                snn_layer_bwd(d, kind, g, xin, self.W[li], self.v[li], self.saved[li],
                              self.gW[li], self.gb[li], self.gv[li], self.gx[li], self.ws, stream)
            if li > 0:
                kind, g = self._grad_below(li)

    def step(self, x, labels=None, targets=None, stream=None):
        self.forward(x, stream)
        self.loss_and_grad(labels, targets, stream)
        self.backward(x, stream)

    def step_fused(self, x, labels=None, targets=None, stream=None):
        """The step as one snn_fused_step launch (needs ``fdesc``): the loss,
        the readout's counts, the hidden spikes and the weight and bias
        gradients land in the buffers ``step`` writes; ``fstatus[0]`` is 0
        after a completed step."""
        if self.fdesc is None:
            raise RuntimeError("step_fused: the library's fused step does not run this network")
        snn_fused_step(self.fdesc, x, self.W[0], self.b[0], self.W[1], self.b[1], labels, targets,
                       self.loss, self.counts, self.gW[0], self.gb[0], self.gW[1], self.gb[1],
                       self.fstatus, self.fws, stream, spk_hidden=self.spk[0])

    def capture_step(self, x, labels=None, targets=None, warmup=2):
        """Capture one forward + loss + BPTT step into a HIP graph (torch's
        CUDAGraph on ROCm) and return it; ``graph.replay()`` then reruns the
        step on the same buffers with one launch from the host.  The library
        records no memset, allocates nothing and never synchronises, so every
        call of the step can be captured."""
        torch = self.torch
        side = torch.cuda.Stream()  # default priority
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(warmup):
                self.step(x, labels, targets)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            self.step(x, labels, targets)
        return graph

    def init_adamw(self, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2):
        """Optimizer state for ``update``: zero moments per parameter tensor
        and, for fp16 weights, an fp32 master copy (the fp16 weights the
        contractions read are rewritten from it after every update)."""
        torch = self.torch
        self.opt = dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay)
        self.opt_t = 0
        self.opt_tensors = []
        for li in range(len(self.descs)):
            for P, G in ((self.W[li], self.gW[li]), (self.b[li], self.gb[li]),
                         (self.v[li], self.gv[li])):
                if P is None:
                    continue
                half = P.dtype == torch.float16
                master = P.float().contiguous() if half else P
                self.opt_tensors.append((master, G, torch.zeros_like(master),
                                         torch.zeros_like(master), P if half else None))

    def update(self, stream=None):
        """One AdamW step over every parameter with the gradients of the last
        backward (Sec. IV: the paper's training step ends with it)."""
        self.opt_t += 1
        snn_adamw(self.opt_tensors, self.opt_t, stream=stream, **self.opt)

    def pool_arg(self, li):
        """The 2x2 pool selection of conv layer li inside its saved buffer
        (None for other layers), at the offset the library reports."""
        return self.parts[li][2]

    # the same work through the stage calls, with a hook between stages
    # (update: finish with the AdamW step of ``init_adamw``; fused_bwd: each
    # layer's backward as one snn_layer_bwd call, hooked as "layer_bwd", as in
    # ``backward``, except for the layers listed in ``staged``).  A dense
    # layer's synapse backward is two stage calls, the weight gradient
    # ("synapse_bwd_dw") then the input gradient ("synapse_bwd_dx"): the same
    # kernels in the same order as one snn_synapse_bwd call with both outputs.
    def step_stages(self, x, labels=None, targets=None, stream=None, hook=None, update=False,
                    fused_bwd=False, staged=()):
        torch = self.torch
        hook = hook or (lambda name, li: None)
        n = len(self.descs)
        h = x
        for li, d in enumerate(self.descs):
            cur, ck, _ = self.parts[li]
            if d.synapse != SYN_NONE:
                hook("synapse_fwd", li)
                snn_synapse_fwd(d, h, self.W[li], self.b[li], cur, self.pool_arg(li), self.ws,
                                stream)
                hook("synapse_fwd_end", li)
            else:
                cur = h
            hook("neuron_fwd", li)
            snn_neuron_fwd(d, cur, self.v[li], self.spk[li], ck,
                           self.counts if li == n - 1 else None, stream)
            hook("neuron_fwd_end", li)
            h = self.spk[li]
        hook("loss", -1)
        self.loss_and_grad(labels, targets, stream)
        hook("loss_end", -1)
        kind, g = GRAD_BCAST, self.gcounts
        for li in range(n - 1, -1, -1):
            d = self.descs[li]
            xin = x if li == 0 else self.spk[li - 1]
            if d.synapse == SYN_NONE:
                hook("neuron_bwd", li)
                snn_neuron_bwd(d, kind, g, self.v[li], xin, self.parts[li][1], self.gx[li], None,
                               self.gv[li], self.ws, stream)
                hook("neuron_bwd_end", li)
                continue
            if fused_bwd and self.dup[li] is None and li not in staged:
                hook("layer_bwd", li)
                snn_layer_bwd(d, kind, g, xin, self.W[li], self.v[li], self.saved[li],
                              self.gW[li], self.gb[li], self.gv[li], self.gx[li], self.ws, stream)
                hook("layer_bwd_end", li)
                if li > 0:
                    kind, g = self._grad_below(li)
                continue
            dcur_bytes = d.T * d.B * d.n_out * (2 if d.grad_dtype in (F16, BF16) else 4)
            if self.dup[li] is not None:
                dcur, rest = self.dup[li], self.ws
            else:
                dcur = self.ws[:dcur_bytes]
                if d.grad_dtype == BF16:
                    dcur = dcur.view(torch.bfloat16)
                elif d.grad_dtype == F16:
                    dcur = dcur.view(torch.float16)
                else:
                    dcur = dcur.view(torch.float32)
                rest = self.ws[(dcur_bytes + 255) // 256 * 256:]
            sc = self.scale[li]
            # the weight gradient's operand written by the scan: transposed
            # (transposed_operand=True; off by default, it measured slower
            # than one transpose, as in the layer call), or the three bf16
            # planes of an fp32 dL/dI in its own layout (always, as in the
            # layer call); the row-major dL/dI only where the input gradient
            # needs it.
            use_t = self.transposed_operand or self.dcur_t_layout[li] == DCUR_T_PLANES
            dt = self.dcur_t if use_t and self.dcur_t_bytes[li] > 0 and \
                self.dup[li] is None else None
            rm = dcur if dt is None or self.gx[li] is not None or self.dup[li] is not None \
                else None
            hook("neuron_bwd", li)
            cur, ck, _ = self.parts[li]
            snn_neuron_bwd(d, kind, g, self.v[li], cur, ck, rm, self.gb[li],
                           self.gv[li], rest, stream, dcur_scale=sc, dcur_t=dt)
            hook("neuron_bwd_end", li)
            if d.synapse == SYN_DENSE:
                hook("synapse_bwd_dw", li)
                snn_synapse_bwd(d, rm, None, xin, self.W[li], self.gW[li], None, rest, stream,
                                dcur_scale=sc, dcur_t=dt)
                hook("synapse_bwd_dw_end", li)
                if self.gx[li] is not None:
                    hook("synapse_bwd_dx", li)
                    snn_synapse_bwd(d, dcur, None, xin, self.W[li], None, self.gx[li], rest,
                                    stream, dcur_scale=sc)
                    hook("synapse_bwd_dx_end", li)
            else:
                hook("synapse_bwd", li)
                snn_synapse_bwd(d, dcur, self.pool_arg(li), xin, self.W[li], self.gW[li],
                                self.gx[li], rest, stream)
                hook("synapse_bwd_end", li)
            if li > 0:
                kind, g = self._grad_below(li)
        if update:
            hook("update", -1)
            self.update(stream)
            hook("update_end", -1)
