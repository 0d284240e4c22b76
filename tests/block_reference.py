"""Plain references of the leaky sequence block's operators in 64 bits (numpy,
token by token and row by row), and the sums of absolute terms that the
tolerances of the GPU tests are stated in."""
import numpy as np

EPS32 = 2.0 ** -24
# half a unit in the last place, relative, and absolute below the type's normal
# range (fp32, bf16: factors under 2^-126 may be flushed; the tests multiply
# them by less than 64)
HALF_ULP = {"f32": (EPS32, 2.0 ** -120), "f16": (2.0 ** -11, 2.0 ** -25),
            "bf16": (2.0 ** -8, 2.0 ** -120)}


def linattn(q, k, v, decay, lens, init, scale):
    """o [T,B,H,dv] and the final state [B,H,dk,dv] of float64 q [T,B,H,dk],
    k, v [T,B,KV,.]."""
    T, B, H, _ = q.shape
    share = H // k.shape[2] if k.shape[2] else 1
    S = init.copy()
    o = np.zeros((T, B, H, v.shape[3]))
    g = decay[:, None, None]
    for t in range(T):
        for b in range(B):
            if t >= lens[b]:
                continue
            kt, vt = (np.repeat(x[t, b], share, axis=0) for x in (k, v))
            S[b] = g * S[b] + kt[:, :, None] * vt[:, None, :]
            o[t, b] = scale * np.einsum("hi,hij->hj", q[t, b], S[b])
    return o, S


def linattn_grads(q, k, v, decay, lens, init, scale, go, gs):
    """dq, dk, dv and the gradient of the initial state, by the reversed recurrence."""
    T, B, H, _ = q.shape
    KV = k.shape[2]
    share = H // KV
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    g = decay[:, None, None]
    S = init.copy()
    for t in range(T):
        for b in range(B):
            if t < lens[b]:
                kt, vt = (np.repeat(x[t, b], share, axis=0) for x in (k, v))
                S[b] = g * S[b] + kt[:, :, None] * vt[:, None, :]
                dq[t, b] = scale * np.einsum("hij,hj->hi", S[b], go[t, b])
    R = gs.copy()
    for t in reversed(range(T)):
        for b in range(B):
            if t < lens[b]:
                kt, vt = (np.repeat(x[t, b], share, axis=0) for x in (k, v))
                full = R[b] + scale * q[t, b][:, :, None] * go[t, b][:, None, :]
                dk[t, b] = np.einsum("hij,hj->hi", full, vt).reshape(KV, share, -1).sum(1)
                dv[t, b] = np.einsum("hij,hi->hj", full, kt).reshape(KV, share, -1).sum(1)
                R[b] = g * full
    return dq, dk, dv, R


def quantised(x, block=128):
    """What an 8-bit checkpoint of fp32 x [rows, n] stands for (its own fp32 steps)."""
    x = np.asarray(x, np.float32)
    out = np.zeros_like(x)
    for a in range(0, x.shape[1], block):
        b = x[:, a:a + block]
        with np.errstate(all="ignore"):
            top = np.abs(b).max(1, keepdims=True)
            fine = np.isfinite(b).all(1, keepdims=True)
            code = np.rint(b * (np.float32(127) / top))
            val = np.where(top >= np.float32(2.0 ** -100), code * (top * np.float32(1 / 127)), 0)
        out[:, a:a + block] = np.where(fine, val, np.nan)
    return out


def _mean(x, groups):
    r, n = x.shape
    m = x.reshape(r, groups, n // groups).mean(2, keepdims=True)
    return np.broadcast_to(m, (r, groups, n // groups)).reshape(r, n)


def gate_norm(x, y, g, groups, act, eps, w_post, scale, w_pre):
    """x_out, h, and the sums of absolute terms of both."""
    if y is None:
        x_out, ax = x, np.abs(x)
    else:
        f, _, _ = gate(act, g)
        u = y / np.sqrt(_mean(y * y, groups) + eps) * w_post
        x_out = x + scale * u * f
        ax = np.abs(x) + np.abs(scale * u * f)
    r = 1 / np.sqrt(_mean(x_out * x_out, 1) + eps)
    # an error of x_out reaches h directly and, averaged, through the root mean square
    ah = r * np.abs(w_pre) * (ax + np.abs(x_out) * r * r * _mean(np.abs(x_out) * ax, 1))
    return x_out, x_out * r * w_pre, ax, ah


def gate(act, g):
    """Factor, slope, and the slope's sum of absolute terms."""
    if act == "none":
        return 1.0, 0.0, 0.0
    if act == "mul":
        return g, np.ones_like(g), np.ones_like(g)
    with np.errstate(over="ignore"):
        p = 1 / (1 + np.exp(-g))
    if act == "sigmoid":
        return p, p * (1 - p), p
    return g * p, p + g * p * (1 - p), p + np.abs(g) * p


def gate_norm_grads(gx, gh, x_out, y, g, groups, act, eps, w_post, scale, w_pre):
    """Gradients and, under "abs_" names, the sums of absolute terms."""
    out = {}
    dx, adx = gx.copy(), np.abs(gx)
    if gh is not None:
        r = 1 / np.sqrt(_mean(x_out * x_out, 1) + eps)
        hat, d = x_out * r, gh * w_pre
        dx = dx + r * (d - hat * _mean(hat * d, 1))
        adx = adx + r * (np.abs(d) + np.abs(hat) * _mean(np.abs(hat * d), 1))
        out["dw_pre"], out["abs_dw_pre"] = (gh * hat).sum(0), np.abs(gh * hat).sum(0)
    out["dx"], out["abs_dx"] = dx, adx
    if y is None:
        return out
    f, slope, aslope = gate(act, g)
    r = 1 / np.sqrt(_mean(y * y, groups) + eps)
    hat = y * r
    da, ada = dx * scale, adx * np.abs(scale)
    dhat, adhat = da * f * w_post, ada * np.abs(f * w_post)
    out["dy"] = r * (dhat - hat * _mean(hat * dhat, groups))
    out["abs_dy"] = r * (adhat + np.abs(hat) * _mean(np.abs(hat) * adhat, groups))
    out["dg"] = da * hat * w_post * slope if g is not None else None
    out["abs_dg"] = ada * np.abs(hat * w_post) * aslope if g is not None else None
    out["dw_post"], out["abs_dw_post"] = (da * f * hat).sum(0), (ada * np.abs(f * hat)).sum(0)
    t = hat * w_post * f
    out["ds"], out["abs_ds"] = (dx * t).sum(0), (adx * np.abs(t)).sum(0)
    return out
