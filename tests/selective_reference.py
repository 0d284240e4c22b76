"""Plain references of the selective leaky block's operators in 64 bits (numpy), token by
token, that carry the error an fp32 computation of the same steps may have.

A ``V`` is a value with a bound of its error.  Every operation adds one fp32 rounding
(2^-24 of the result) to what its operands bring; a function of the kernels adds a few:
exponential, softplus and sigmoid up to 8 units.  A sum of n terms in any order adds n
units of the sum of their absolute values."""
import numpy as np

U = 2.0 ** -24
FEW = 8 * U
# half a unit in the last place, relative, and absolute below the type's normal range
HALF_ULP = {"f32": (U, 2.0 ** -120), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 2.0 ** -120)}


class V:
    def __init__(self, v, e=0.0):
        self.v = np.asarray(v, np.float64)
        self.e = np.broadcast_to(np.asarray(e, np.float64), self.v.shape)

    def __add__(self, o):
        o = o if isinstance(o, V) else V(o)
        s = self.v + o.v
        return V(s, self.e + o.e + U * np.abs(s))

    def __mul__(self, o):
        o = o if isinstance(o, V) else V(o)
        s = self.v * o.v
        return V(s, np.abs(self.v) * o.e + np.abs(o.v) * self.e + self.e * o.e + U * np.abs(s))

    def __getitem__(self, i):
        return V(self.v[i], self.e[i])

    def sum(self, axis):
        n = np.prod([self.v.shape[a] for a in np.atleast_1d(axis)]) if self.v.size else 0
        axis = tuple(np.atleast_1d(axis))
        return V(self.v.sum(axis), self.e.sum(axis) + n * U * np.abs(self.v).sum(axis))

    def where(self, on, other=0.0):
        o = other if isinstance(other, V) else V(np.broadcast_to(other, self.v.shape))
        return V(np.where(on, self.v, o.v), np.where(on, self.e, o.e))


def exp(x):
    r = np.exp(x.v)
    return V(r, r * np.expm1(np.minimum(x.e, 1.0)) + FEW * r)


def softplus(x):
    r = np.logaddexp(0.0, x.v)
    return V(r, sigmoid(x).v * x.e + FEW * r)


def sigmoid(x):
    r = 1 / (1 + np.exp(-x.v))
    return V(r, r * (1 - r) * x.e + FEW * r)


def silu(z):
    """The factor and its slope, each with the sum of its terms as rounding's scale."""
    p = 1 / (1 + np.exp(-z))
    return V(z * p, FEW * np.abs(z * p)), V(p + z * p * (1 - p),
                                            FEW * (p + np.abs(z) * p * (1 - p)))


def stack(xs, shape):
    if not xs:
        return V(np.zeros((0,) + shape))
    return V(np.stack([x.v for x in xs]), np.stack([x.e for x in xs]))


def selscan(u, dt, a, b, c, skip, dt_bias, z, lens, init, soft=True, gy=None, gs=None):
    """float64 u, dt, z [T,B,n], a [N,n], b, c [T,B,G,N], init [B,N,n]: y and the state,
    and with gy and gs a dictionary of gradients (all V)."""
    T, B, n = u.shape
    G = b.shape[2]
    group = np.arange(n) // max(n // G, 1)
    per = [np.arange(T)[t] < lens for t in range(T)]
    wide = [np.transpose(x[:, :, group], (0, 1, 3, 2)) for x in (b, c)]  # [T,B,N,n]

    def token(t):
        on = per[t][:, None]
        raw = V(np.where(on, dt[t], 0.0)) + dt_bias
        d = (softplus(raw) if soft else raw).where(on)
        ut = np.where(on, u[t], 0.0)
        bt, ct = (np.where(on[:, None], x[t], 0.0) for x in wide)
        e = exp(V(d.v[:, None], d.e[:, None]) * a)
        return on, raw, d, ut, bt, ct, e

    hs, ys, ins = [V(init)], [], []
    for t in range(T):
        on, raw, d, ut, bt, ct, e = token(t)
        du = d * ut
        h = (e * hs[-1] + V(du.v[:, None], du.e[:, None]) * bt).where(on[:, None], hs[-1])
        inner = (h * ct).sum(1) + V(ut) * skip
        y = inner * silu(np.where(on, z[t], 0.0))[0] if z is not None else inner
        hs.append(h)
        ins.append(inner)
        ys.append(y.where(on))
    y = stack(ys, (B, n))
    if gy is None:
        return y, hs[-1]
    R, out = V(gs), {k: [] for k in ("du", "ddt", "db", "dc", "dz")}
    da, dskip, dbias = [], [], []

    def by_group(x):  # [B,N,n] -> [B,G,N]
        parts = [V(x.v[:, :, group == g], x.e[:, :, group == g]).sum(2) for g in range(G)]
        return V(np.stack([p.v for p in parts], 1), np.stack([p.e for p in parts], 1))

    for t in reversed(range(T)):
        on, raw, d, ut, bt, ct, e = token(t)
        g = np.where(on, gy[t], 0.0)
        gi = V(g)
        if z is not None:
            act, slope = silu(np.where(on, z[t], 0.0))
            gi = act * g
            out["dz"].insert(0, (slope * g * ins[t]).where(on))
        wide_gi = V(gi.v[:, None], gi.e[:, None])
        full = wide_gi * ct + R
        du = d * ut
        out["dc"].insert(0, by_group((wide_gi * hs[t + 1]).where(on[:, None])))
        out["db"].insert(0, by_group((full * V(du.v[:, None], du.e[:, None])).where(on[:, None])))
        gin = (full * bt).sum(1)
        ge = (e * full * hs[t])
        gd = gin * ut + (ge * a).sum(1)
        gdt = (gd * sigmoid(raw) if soft else gd).where(on)
        out["du"].insert(0, (gin * d + gi * skip).where(on))
        out["ddt"].insert(0, gdt)
        da.append((ge * V(d.v[:, None], d.e[:, None])).where(on[:, None]))
        dskip.append(gi * ut)
        dbias.append(gdt)
        R = (e * full).where(on[:, None], R)
    shapes = dict(du=(B, n), ddt=(B, n), dz=(B, n), db=(B,) + b.shape[2:], dc=(B,) + b.shape[2:])
    out = {k: stack(v, shapes[k]) for k, v in out.items()}
    if z is None:
        del out["dz"]
    out["da"] = stack(da, (B,) + a.shape).sum((0, 1))
    out["dskip"] = stack(dskip, (B, n)).sum((0, 1))
    out["dbias"] = stack(dbias, (B, n)).sum((0, 1))
    out["dstate"] = R
    return y, hs[-1], out


def shortconv(x, w, bias, lens, init, act, gy=None, gs=None):
    """float64 x [T,B,n], w [K,n], init [B,K-1,n]: y and the state, and with gy and gs the
    gradients (all V)."""
    T, B, n = x.shape
    K = w.shape[0]
    y, ye = np.zeros((T, B, n)), np.zeros((T, B, n))
    state = np.zeros((B, K - 1, n))
    dx, dxe = np.zeros((T, B, n)), np.zeros((T, B, n))
    ds, dse = np.zeros((B, K - 1, n)), np.zeros((B, K - 1, n))
    dw, dwa, db, dba = (np.zeros(s) for s in ((K, n), (K, n), (n,), (n,)))
    for i in range(B):
        m = lens[i]
        seen = np.concatenate([init[i], x[:m, i]])
        state[i] = seen[m:]
        pre = sum((w[j] * seen[j:j + m] for j in range(K)), bias + np.zeros((m, n)))
        size = sum((np.abs(w[j] * seen[j:j + m]) for j in range(K)), np.abs(bias) + np.zeros((m, n)))
        pe = (K + 2) * U * size
        f, slope = silu(pre) if act == "silu" else (V(pre), V(np.ones_like(pre)))
        # the slope of silu is at most 1.1, its curvature at most 0.5
        y[:m, i], ye[:m, i] = f.v, f.e + 1.1 * pe
        if gy is None:
            continue
        g = gy[:m, i] * slope.v
        ge = np.abs(gy[:m, i]) * (slope.e + (0.5 * pe if act == "silu" else 0.0)) + U * np.abs(g)
        acc, ae = np.zeros((m + K - 1, n)), np.zeros((m + K - 1, n))
        for j in range(K):
            acc[j:j + m] += w[j] * g
            ae[j:j + m] += np.abs(w[j]) * (ge + (K + 2) * U * np.abs(g))
            dw[j] += (g * seen[j:j + m]).sum(0)
            dwa[j] += ((ge + (T * B + 2) * U * np.abs(g)) * np.abs(seen[j:j + m])).sum(0)
        acc[m:] += gs[i]
        ae[m:] += (K + 2) * U * np.abs(gs[i])
        db += g.sum(0)
        dba += (ge + (T * B + 2) * U * np.abs(g)).sum(0)
        dx[:m, i], dxe[:m, i], ds[i], dse[i] = acc[K - 1:], ae[K - 1:], acc[:K - 1], ae[:K - 1]
    if gy is None:
        return V(y, ye), state
    return V(y, ye), state, dict(dx=V(dx, dxe), dw=V(dw, dwa), dbias=V(db, dba), dstate=V(ds, dse))


def layer_norm(x, w, b, eps, gy=None, gres=None):
    """float64 x [R,n]: y, and with gy the gradients (all V).  The sums over a row are a
    tree of at most 16 + log2(1024) levels; 64 units of the sums of absolute terms cover
    them and the operations on their results."""
    C = 64 * U
    n = x.shape[1]
    size = np.abs(x) + np.abs(x).mean(1, keepdims=True)  # terms of x - mean
    mid = x - x.mean(1, keepdims=True)
    r = 1 / np.sqrt((mid * mid).mean(1, keepdims=True) + eps)
    hat = mid * r
    # errors of mid reach r through the mean square, halved and averaged
    hat_size = r * (size + np.abs(hat) * (np.abs(hat) * size).mean(1, keepdims=True) + np.abs(mid))
    y = V(hat * w + b, C * (np.abs(w) * hat_size + np.abs(b)))
    if gy is None:
        return y
    g = gy * w
    r_size = (np.abs(hat) * size).mean(1, keepdims=True) * r + 1  # of r, relative
    mg, mh = g.mean(1, keepdims=True), (g * hat).mean(1, keepdims=True)
    dx = gres + r * (g - mg - hat * mh)
    terms = np.abs(g) + np.abs(g).mean(1, keepdims=True) + hat_size * np.abs(mh) + \
        np.abs(hat) * (np.abs(g) * (hat_size + np.abs(hat))).mean(1, keepdims=True)
    dxe = C * (np.abs(gres) + r * (terms + np.abs(g - mg - hat * mh) * r_size))
    rows = x.shape[0]
    dw = V((gy * hat).sum(0), (C * np.abs(gy) * hat_size).sum(0) +
           (rows + 2) * U * np.abs(gy * hat).sum(0))
    db = V(gy.sum(0), (rows + 2) * U * np.abs(gy).sum(0))
    return y, dict(dx=V(dx, dxe), dw=dw, db=db)


def near(got, want, dt, what=""):
    """Within twice the carried error (orders and joins of sums other than the
    reference's) and half a unit of the type."""
    got = np.asarray(got, np.float64)
    assert got.shape == want.v.shape, (what, got.shape, want.v.shape)
    rel, least = HALF_ULP[dt]
    bound = 2 * want.e + rel * (np.abs(want.v) + 2 * want.e) + least
    assert np.isfinite(got).all(), what
    err = np.abs(got - want.v)
    assert (err <= bound).all(), (what, float((err / bound).max()),
                                  np.unravel_index((err / bound).argmax(), err.shape))
