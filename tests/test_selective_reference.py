"""The 64-bit references of the selective leaky block against differences: each gradient
is that of a weighted sum of the outputs (no GPU needed)."""
import numpy as np
import pytest

from tests import selective_reference as ref


def _check(f, args, grads, rng, skip=()):
    """f(*args) -> scalar; grads: one per argument, by central differences of 1e-5, whose
    error is 1e-10 of a third derivative and 1e-11 of rounding."""
    for k, (x, g) in enumerate(zip(args, grads)):
        if g is None:
            continue
        g = g.v
        for _ in range(12):
            i = tuple(rng.integers(0, s) for s in x.shape)
            up, down = x.copy(), x.copy()
            up[i] += 1e-5
            down[i] -= 1e-5
            d = (f(*args[:k], up, *args[k + 1:]) - f(*args[:k], down, *args[k + 1:])) / 2e-5
            assert abs(d - g[i]) <= 1e-6 * (1 + abs(g[i])), (k, i, d, g[i])


@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("soft", [True, False])
def test_selscan(gate, soft):
    rng = np.random.default_rng(3)
    T, B, n, N, G = 7, 3, 6, 3, 2
    lens = np.array([7, 0, 4])
    u, dt, z, gy = (rng.standard_normal((T, B, n)) for _ in range(4))
    dt = dt if soft else 0.3 + 0.1 * np.abs(dt)
    a, (b, c) = -np.exp(rng.standard_normal((N, n))), rng.standard_normal((2, T, B, G, N))
    skip, bias = rng.standard_normal((2, n))
    bias = bias if soft else 0.1 * np.abs(bias)
    init, gs = rng.standard_normal((2, B, N, n))
    args = [u, dt, a, b, c, skip, bias, z, init]

    def run(u, dt, a, b, c, skip, bias, z, init, **more):
        return ref.selscan(u, dt, a, b, c, skip, bias, z if gate else None, lens, init, soft,
                           **more)

    def f(*x):
        y, s = run(*x)
        return (y.v * gy).sum() + (s.v * gs).sum()

    g = run(*args, gy=gy, gs=gs)[2]
    _check(f, args, [g["du"], g["ddt"], g["da"], g["db"], g["dc"], g["dskip"], g["dbias"],
                     g.get("dz"), g["dstate"]], rng)


@pytest.mark.parametrize("act", ["none", "silu"])
def test_shortconv(act):
    rng = np.random.default_rng(4)
    T, B, n, K = 6, 4, 5, 4
    lens = np.array([6, 0, 2, 3])
    x, gy = rng.standard_normal((2, T, B, n))
    w, bias = rng.standard_normal((K, n)), rng.standard_normal(n)
    init, gs = rng.standard_normal((2, B, K - 1, n))

    def f(x, w, bias, init):
        y, s = ref.shortconv(x, w, bias, lens, init, act)
        return (y.v * gy).sum() + (s * gs).sum()

    g = ref.shortconv(x, w, bias, lens, init, act, gy, gs)[2]
    _check(f, [x, w, bias, init], [g["dx"], g["dw"], g["dbias"], g["dstate"]], rng)


def test_layer_norm():
    rng = np.random.default_rng(5)
    x, gy = rng.standard_normal((2, 5, 9))
    w, b = rng.standard_normal((2, 9))

    def f(x, w, b):
        return (ref.layer_norm(x, w, b, 1e-3).v * gy).sum()

    g = ref.layer_norm(x, w, b, 1e-3, gy, np.zeros_like(x))[1]
    _check(f, [x, w, b], [g["dx"], g["dw"], g["db"]], rng)
