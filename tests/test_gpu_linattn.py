"""Linear attention with a decay per head against the recurrence in 64 bits.

Tolerance, per element: with A the same expression on absolute values (the sum
of the absolute values of all terms), fp32 accumulation of at most d + T
products in any order with a few roundings of each factor errs by at most
(d + T + 24) 2^-24 A; a 16-bit kernel may hold a score or the state as two
16-bit parts, 2^-16 A for both together; the result's own rounding adds half a
unit in its last place.  Gradients of shared heads sum that many terms more."""
import numpy as np
import pytest

import paper_2211_10725_amd as snn
from tests import block_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _rand(rng, shape, dt, std=1.0):
    x = torch.as_tensor(rng.standard_normal(shape) * std, dtype=torch.float32)
    return x.to(TYPES[dt]).cuda()


def _np(x):
    return x.detach().double().cpu().numpy()


def _empty_like(x):
    """NaN-filled tensor of the same strides."""
    out = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)
    return out.fill_(float("nan"))


class Case:
    def __init__(self, T, B, H, KV, dk, dv, dt, lens=None, packed=False, order=None, decay=None,
                 seed=0, state=True, std=1.0):
        rng = np.random.default_rng(seed)
        self.dt, self.scale, self.shape = dt, dk ** -0.5, (T, B, H, KV, dk, dv)
        w = [H * dk, KV * dk, KV * dv]
        if packed:
            parts = _rand(rng, (T, B, sum(w) + 8), dt, std)[:, :, 8:].split(w, dim=2)
            self.q, self.k, self.v = (p.unflatten(2, (-1, d)) for p, d in zip(parts, (dk, dk, dv)))
        else:
            def tensor(h, d):
                x = _rand(rng, (T, B, h, d), dt, std)
                if order:  # another order in memory, the same indices
                    perm = [list(order).index(i) for i in range(3)]
                    x = x.permute(*order, 3).contiguous().permute(*perm, 3)
                return x
            self.q, self.k, self.v = tensor(H, dk), tensor(KV, dk), tensor(KV, dv)
        g = np.linspace(0.5, 0.998, H) if decay is None else np.resize(decay, H)
        self.decay = torch.as_tensor(g, dtype=torch.float32).cuda()
        self.lens = None if lens is None else torch.as_tensor(lens, dtype=torch.int32).cuda()
        self.n = [T] * B if lens is None else [min(max(int(x), 0), T) for x in lens]
        self.s0 = _rand(rng, (B, H, dk, dv), "f32") if state else None
        self.go = _rand(rng, (T, B, H, dv), dt, std)
        self.gs = _rand(rng, (B, H, dk, dv), "f32") if state else None
        self.o = torch.full((T, B, H, dv), float("nan"), dtype=TYPES[dt], device="cuda")
        self.d = snn.linattn_desc(self.q, self.k, self.v, self.o, self.scale)
        self.ws = torch.empty(max(16, snn.snn_linattn_workspace_bytes(self.d)),
                              dtype=torch.uint8, device="cuda")

    def fwd(self, state_out=None, s0="own"):
        self.s = torch.full((self.shape[1], self.shape[2], *self.shape[4:]), float("nan"),
                            device="cuda") if state_out is None else state_out
        snn.snn_linattn_fwd(self.d, self.q, self.k, self.v, self.decay, self.lens,
                            self.s0 if isinstance(s0, str) else s0, self.o, self.s, self.ws)
        return self.o, self.s

    def bwd(self):
        self.dq, self.dk, self.dv = (_empty_like(x) for x in (self.q, self.k, self.v))
        self.ds = torch.full_like(self.gs, float("nan")) if self.gs is not None else \
            torch.full((self.shape[1], self.shape[2], *self.shape[4:]), float("nan"),
                       device="cuda")
        snn.snn_linattn_bwd(self.d, self.q, self.k, self.v, self.decay, self.lens, self.s0,
                            self.go, self.gs, self.dq, self.dk, self.dv, self.ds, self.ws)
        return self.dq, self.dk, self.dv, self.ds

    def _zero_state(self):
        T, B, H, KV, dk, dv = self.shape
        return np.zeros((B, H, dk, dv))

    def arrays(self, f=lambda x: x):
        z = self._zero_state()
        return [f(_np(x)) for x in (self.q, self.k, self.v, self.decay)] + \
            [self.n, f(_np(self.s0)) if self.s0 is not None else z, self.scale]

    def tol(self, got, want, absolute, fp32=False):
        T, B, H, KV, dk, dv = self.shape
        terms = max(dk, dv) + T + 24 + H // max(KV, 1)
        rel, least = ref.HALF_ULP["f32" if fp32 else self.dt]
        parts = 0.0 if self.dt == "f32" or fp32 else 2.0 ** -16
        bound = (terms * ref.EPS32 + parts) * absolute + rel * np.abs(want) + least
        err = np.abs(got - want)
        assert np.isfinite(got).all()
        assert (err <= bound).all(), (self.shape, self.dt, float((err / bound).max()))

    def check_fwd(self):
        o, s = self.fwd()
        wo, ws = ref.linattn(*self.arrays())
        ao, as_ = ref.linattn(*self.arrays(np.abs))
        self.tol(_np(o), wo, ao)
        self.tol(_np(s), ws, as_, fp32=True)
        for b, n in enumerate(self.n):
            assert (o[n:, b] == 0).all()

    def check_bwd(self):
        got = self.bwd()
        z = self._zero_state()
        go, gs = _np(self.go), _np(self.gs) if self.gs is not None else z
        want = ref.linattn_grads(*self.arrays(), go, gs)
        absolute = ref.linattn_grads(*self.arrays(np.abs), np.abs(go), np.abs(gs))
        for i, (g, w, a) in enumerate(zip(got, want, absolute)):
            self.tol(_np(g), w, a, fp32=i == 3)
        for b, n in enumerate(self.n):
            for g in got[:3]:
                assert (g[n:, b] == 0).all()


# (T, B, H, KV, dk, dv): one token to several chunks and segments, odd counts,
# head sizes that fill no tile, shared heads
SIZES = [(1, 1, 1, 1, 8, 8), (2, 3, 2, 2, 16, 8), (15, 1, 3, 1, 24, 40), (16, 2, 2, 2, 64, 64),
         (17, 2, 2, 1, 64, 32), (31, 1, 1, 1, 128, 128), (32, 1, 2, 2, 32, 128),
         (33, 2, 3, 3, 72, 104), (63, 1, 2, 2, 64, 64), (64, 2, 1, 1, 128, 64),
         (65, 1, 4, 2, 40, 72), (127, 2, 2, 2, 32, 32), (129, 3, 2, 1, 96, 80),
         (200, 1, 6, 3, 64, 64), (257, 2, 2, 2, 128, 128), (700, 1, 2, 2, 64, 64)]


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward_and_backward(size, dt):
    c = Case(*size, dt, seed=sum(size))
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("dt", list(TYPES))
def test_without_states(dt):
    c = Case(70, 2, 2, 2, 64, 48, dt, state=False)
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("lens", [[0, 1, 64, 150], [150, 0, 0, 65], [-3, 2, 900, 128]])
def test_ragged_lengths_and_empty_rows(lens, dt):
    c = Case(150, 4, 2, 1, 64, 72, dt, lens=lens)
    for b, n in enumerate(c.n):  # what is past the end is never read
        for x in (c.q, c.k, c.v, c.go):
            x[n:, b] = float("nan")
    z = [torch.nan_to_num(x, nan=0.0) for x in (c.q, c.k, c.v, c.go)]
    c.fwd(), c.bwd()
    got = [x.clone() for x in (c.o, c.s, c.dq, c.dk, c.dv, c.ds)]
    c.q, c.k, c.v, c.go = z
    c.check_fwd(), c.check_bwd()
    for a, b in zip(got, (c.o, c.s, c.dq, c.dk, c.dv, c.ds)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("order", [(1, 0, 2), (2, 1, 0), (1, 2, 0)])
def test_orders_in_memory(order, dt):
    c = Case(75, 3, 2, 2, 40, 64, dt, order=order)
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("dt", list(TYPES))
def test_slices_of_a_packed_projection(dt):
    c = Case(90, 2, 4, 2, 64, 48, dt, packed=True)
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("decay", [[0.0], [1.0], [0.0, 1e-30, 0.3, 1.0], [-0.7, 1.01]])
def test_decays(decay, dt):
    c = Case(140, 1, 4, 4, 32, 64, dt, decay=decay)
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("std", [1e-3, 60.0])
def test_small_and_large_values(std, dt):
    # 60^2 x 128 tokens: scores and states far above fp16's largest value
    c = Case(160, 1, 2, 2, 64, 64, dt, std=std, decay=[1.0, 0.99])
    c.scale = 1e-4 if std > 1 else 1.0
    c.d = snn.linattn_desc(c.q, c.k, c.v, c.o, c.scale)
    c.check_fwd()
    if dt != "f16" or std < 1:  # its gradients leave fp16's range
        c.check_bwd()


def test_large_states_half():
    """Sums of fp16 products above 65504 inside: scores and states stay right."""
    c = Case(200, 1, 1, 1, 64, 64, "f16", decay=[1.0], state=False)
    c.q.fill_(30.0), c.k.fill_(30.0), c.v.fill_(20.0)
    c.scale = 1e-4
    c.d = snn.linattn_desc(c.q, c.k, c.v, c.o, c.scale)
    c.check_fwd()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("what", ["v", "k", "q"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_later_tokens_never_reach_earlier_outputs(what, value, dt):
    c = Case(150, 1, 1, 1, 64, 64, dt)
    at = 75
    getattr(c, what)[at, 0, 0, 5] = value
    o, s = c.fwd()
    assert torch.isfinite(o[:at]).all()
    assert not torch.isfinite(o[at]).all()
    wo, _ = ref.linattn(*[np.nan_to_num(x, nan=0, posinf=0) if isinstance(x, np.ndarray) else x
                          for x in c.arrays()])
    ao, _ = ref.linattn(*[np.abs(np.nan_to_num(x, nan=0, posinf=0))
                          if isinstance(x, np.ndarray) else x for x in c.arrays()])
    cut = Case(150, 1, 1, 1, 64, 64, dt)
    cut.tol(_np(o[:at]), wo[:at], ao[:at])
    if what == "q":  # its own output alone
        assert torch.isfinite(o[at + 1:]).all() and torch.isfinite(s).all()
    else:
        assert not torch.isfinite(o[-1]).all() and not torch.isfinite(s).all()
    if what == "v":  # the other columns of v stay finite
        keep = [i for i in range(64) if i != 5]
        assert torch.isfinite(o[:, :, :, keep]).all() and torch.isfinite(s[..., keep]).all()


@pytest.mark.parametrize("dt", list(TYPES))
def test_infinities_leave_other_columns_and_tokens_as_they_were(dt):
    """Values far above fp16's range inside (scores and states to 1e6), cut into
    segments: an infinity in one column of v, and one in a late k, change nothing
    of the other columns and of the tokens before."""
    c = Case(1100, 1, 1, 1, 64, 64, dt, std=40.0, decay=[0.9])
    c.scale = 1e-4
    c.d = snn.linattn_desc(c.q, c.k, c.v, c.o, c.scale)
    wo, ws = ref.linattn(*c.arrays())
    ao, as_ = ref.linattn(*c.arrays(np.abs))
    keep = [i for i in range(64) if i != 9]
    old = c.v[40, 0, 0, 9].item()
    c.v[40, 0, 0, 9] = float("inf")
    o, s = c.fwd()
    c.tol(_np(o)[..., keep], wo[..., keep], ao[..., keep])
    c.tol(_np(s)[..., keep], ws[..., keep], as_[..., keep], fp32=True)
    c.v[40, 0, 0, 9] = old
    c.k[1090, 0, 0, 3] = float("inf")
    o, s = c.fwd()
    c.tol(_np(o[:1090]), wo[:1090], ao[:1090])
    assert not torch.isfinite(o[1090:]).any()
    rows = [i for i in range(64) if i != 3]
    c.tol(_np(s)[:, :, rows], ws[:, :, rows], as_[:, :, rows], fp32=True)


@pytest.mark.parametrize("dt", list(TYPES))
def test_state_carries_over_calls_and_in_place(dt):
    c = Case(130, 2, 2, 1, 64, 64, dt)
    whole, end = (x.clone() for x in c.fwd())
    state = c.s0.clone()
    outs = []
    for a, b in ((0, 1), (1, 50), (50, 130)):
        o = torch.empty_like(c.o[a:b])
        d = snn.linattn_desc(c.q[a:b], c.k[a:b], c.v[a:b], o, c.scale)
        ws = torch.empty(max(16, snn.snn_linattn_workspace_bytes(d)), dtype=torch.uint8,
                         device="cuda")
        snn.snn_linattn_fwd(d, c.q[a:b], c.k[a:b], c.v[a:b], c.decay, None, state, o, state, ws)
        outs.append(o)
    wo, ws_ = ref.linattn(*c.arrays())
    ao, as_ = ref.linattn(*c.arrays(np.abs))
    c.tol(_np(torch.cat(outs)), wo, ao)
    c.tol(_np(state), ws_, as_, fp32=True)
    c.tol(_np(whole), wo, ao)
    c.tol(_np(end), ws_, as_, fp32=True)


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,d", [(300, 64), (700, 64), (1500, 128)])
def test_state_in_place_over_many_segments(T, d, dt):
    """One head: the tokens are cut into segments, with the state given, in place,
    apart and absent."""
    c = Case(T, 1, 1, 1, d, d, dt, lens=[T - 70])
    o, s = (x.clone() for x in c.fwd())
    c.check_fwd()
    state = c.s0.clone()
    c.fwd(state_out=state, s0=state)
    assert torch.equal(c.o, o) and torch.equal(state, s)
    c.check_bwd()
    z = Case(T, 1, 1, 1, d, d, dt, state=False)
    z.check_fwd()
    z.check_bwd()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,B,H,KV,dk,dv", [(20, 65, 4, 2, 128, 72), (640, 33, 2, 1, 72, 40),
                                            (1152, 15, 2, 2, 72, 72), (1152, 5, 2, 1, 40, 72),
                                            (40, 150, 7, 7, 16, 24)])
def test_more_workgroups_than_compute_units(T, B, H, KV, dk, dv, dt):
    """Many heads, uncut and in segments of a few hundred tokens."""
    c = Case(T, B, H, KV, dk, dv, dt, lens=[T - (b % 3) * T // 2 for b in range(B)])
    c.check_fwd()
    c.check_bwd()


def test_no_tokens_and_no_sequences():
    for T, B, H, KV in ((0, 2, 2, 2), (5, 0, 2, 2)):
        c = Case(T, B, H, KV, 64, 64, "bf16")
        o, s = c.fwd()
        dq, dk, dv, ds = c.bwd()
        assert torch.equal(s, c.s0) and torch.equal(ds, c.gs)
    c = Case(0, 2, 2, 2, 64, 64, "f32", state=False)
    o, s = c.fwd()
    assert (s == 0).all()


@pytest.mark.parametrize("dt", list(TYPES))
def test_gradient_against_differences(dt):
    """The loss <o, go> + <S, gs> is linear in each of q, k, v and the first
    state, so a difference of the kernel's own losses is the gradient's product
    with the step, whatever the step: fp32 inputs; in 16 bits the outputs'
    rounding of 2^-8 of each term bounds it."""
    c = Case(100, 2, 2, 1, 64, 72, dt, lens=[100, 37])
    grads = [_np(g) for g in c.bwd()]
    live = np.zeros((100, 2, 1, 1))
    for b, n in enumerate(c.n):
        live[:n, b] = 1

    def loss():
        o, s = c.fwd()
        terms = (_np(o) * _np(c.go) * live, _np(s) * _np(c.gs))
        return sum(t.sum() for t in terms), sum(np.square(t).sum() for t in terms)

    base, sq = loss()
    rng = np.random.default_rng(5)
    for name, g in zip(("q", "k", "v", "s0"), grads):
        x = getattr(c, name)
        old = x.clone()
        # a step that the type holds exactly, beside the values
        step = torch.as_tensor(rng.integers(-1, 2, x.shape) * 0.5, dtype=x.dtype, device="cuda")
        x.copy_((old + step).to(x.dtype))
        moved = _np(x) - _np(old)
        new, sq2 = loss()
        x.copy_(old)
        want = float((np.nan_to_num(g) * moved).sum())
        # independent roundings of the terms of both losses and of the gradient
        unit = 2.0 ** -8 if dt == "bf16" else 2.0 ** -11 if dt == "f16" else 300 * ref.EPS32
        spread = np.sqrt(sq + sq2 + np.square(np.nan_to_num(g) * moved).sum())
        assert abs((new - base) - want) <= 6 * unit * spread, (name, new - base, want)


def test_runs_are_identical():
    for dt in TYPES:
        c = Case(600, 2, 4, 2, 128, 64, dt, packed=True)
        first = [x.clone() for x in (*c.fwd(), *c.bwd())]
        for a, b in zip(first, (*c.fwd(), *c.bwd())):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("size", [(1, 1, 1, 8, 8), (3, 4, 2, 64, 64), (5, 6, 6, 72, 40),
                                  (2, 8, 1, 128, 128), (70, 3, 3, 24, 104)])
def test_step_against_recurrence(size, dt):
    B, H, KV, dk, dv = size
    c = Case(1, B, H, KV, dk, dv, dt, packed=True)
    pool = torch.full((B + 3, H, dk, dv), 7.0, device="cuda")
    slots = torch.as_tensor(np.random.default_rng(1).permutation(B + 3)[:B], dtype=torch.int32)
    pool[slots.long().cuda()] = c.s0
    kept = pool.clone()
    out = torch.full_like(pool, 9.0)
    snn.snn_linattn_step(c.d, c.q, c.k, c.v, c.decay, slots.cuda(), pool, out, c.o)
    wo, ws = ref.linattn(*c.arrays())
    ao, as_ = ref.linattn(*c.arrays(np.abs))
    c.tol(_np(c.o), wo, ao)
    c.tol(_np(out[slots.long().cuda()]), ws, as_, fp32=True)
    rest = [i for i in range(B + 3) if i not in slots.tolist()]
    assert torch.equal(pool, kept) and (out[rest] == 9.0).all()
    o = c.o.clone()
    snn.snn_linattn_step(c.d, c.q, c.k, c.v, c.decay, slots.cuda(), pool, pool, c.o)  # in place
    assert torch.equal(o, c.o) and torch.equal(pool[slots.long().cuda()],
                                               out[slots.long().cuda()])
    assert (pool[rest] == 7.0).all()
    # no slots: request b in slot b
    snn.snn_linattn_step(c.d, c.q, c.k, c.v, c.decay, None, c.s0, c.s0, c.o)
    assert torch.equal(o, c.o) and torch.equal(c.s0, out[slots.long().cuda()])


def test_idle_requests_touch_nothing():
    c = Case(1, 4, 2, 2, 64, 64, "f16")
    slots = torch.as_tensor([-1, 1, 5, 0], dtype=torch.int32).cuda()
    pool = c.s0.clone()
    snn.snn_linattn_step(c.d, c.q, c.k, c.v, c.decay, slots, pool, pool, c.o)
    assert (c.o[0, 0] == 0).all() and (c.o[0, 2] == 0).all() and (c.o[0, 1] != 0).any()
    assert torch.equal(pool[2:], c.s0[2:]) and not torch.equal(pool[:2], c.s0[:2])


def test_tokens_one_by_one_are_the_prompt():
    c = Case(40, 2, 4, 2, 64, 64, "f32")
    o, s = c.fwd()
    state = c.s0.clone()
    rows = []
    for t in range(40):
        row = torch.empty_like(c.o[:1])
        d = snn.linattn_desc(c.q[t:t + 1], c.k[t:t + 1], c.v[t:t + 1], row, c.scale)
        snn.snn_linattn_step(d, c.q[t:t + 1], c.k[t:t + 1], c.v[t:t + 1], c.decay, None, state,
                             state, row)
        rows.append(row)
    ao, as_ = ref.linattn(*c.arrays(np.abs))
    c.tol(_np(torch.cat(rows)), _np(o), 2 * ao)
    c.tol(_np(state), _np(s), 2 * as_, fp32=True)


def test_offsets_past_32_bits():
    # a pool whose last states lie past 2^31 elements
    H, slots = 16, 8200
    c = Case(1, 2, H, H, 128, 128, "f32")
    pool = torch.empty((slots, H, 128, 128), device="cuda")
    at = torch.as_tensor([slots - 1, 3], dtype=torch.int32).cuda()
    pool[at.long()] = c.s0
    snn.snn_linattn_step(c.d, c.q, c.k, c.v, c.decay, at, pool, pool, c.o)
    wo, ws = ref.linattn(*c.arrays())
    ao, as_ = ref.linattn(*c.arrays(np.abs))
    c.tol(_np(c.o), wo, ao)
    c.tol(_np(pool[at.long()]), ws, as_, fp32=True)
    del pool
    # tokens 2^26 elements apart: the last start past 2^32 elements
    small = Case(66, 1, 1, 1, 64, 64, "bf16")
    big = torch.empty(66 * 2 ** 26 + 64, dtype=torch.bfloat16, device="cuda")
    far = [torch.as_strided(big, (66, 1, 1, 64), (2 ** 26, 64, 64, 1), 64 * i) for i in range(5)]
    for f, x in zip(far[:3], (small.q, small.k, small.v)):
        f.copy_(x)
    small.o = far[3]
    small.q, small.k, small.v = far[:3]
    small.d = snn.linattn_desc(*far[:4], small.scale)
    small.check_fwd()
    far[4].copy_(small.go)
    small.go = far[4]
    small.bwd = lambda: _grads_into(small, far)
    want = ref.linattn_grads(*small.arrays(), _np(small.go), _np(small.gs))
    absolute = ref.linattn_grads(*small.arrays(np.abs), np.abs(_np(small.go)),
                                 np.abs(_np(small.gs)))
    for i, (g, w, a) in enumerate(zip(small.bwd(), want, absolute)):
        small.tol(_np(g), w, a, fp32=i == 3)


def _grads_into(c, far):
    """Gradients into views further along in the same memory as the inputs."""
    big = far[0]
    out = [torch.as_strided(big, (66, 1, 1, 64), (2 ** 26, 64, 64, 1), 64 * (8 + i))
           for i in range(3)]
    ds = torch.empty_like(c.gs)
    d = snn.linattn_desc(c.q, c.k, c.v, c.go, c.scale)
    snn.snn_linattn_bwd(d, c.q, c.k, c.v, c.decay, None, c.s0, c.go, c.gs, *out, ds, c.ws)
    return (*out, ds)


def test_on_another_stream_and_in_a_graph():
    c = Case(300, 2, 4, 2, 64, 64, "bf16")
    want = [x.clone() for x in (*c.fwd(), *c.bwd())]
    for x in (c.o, c.s, c.dq, c.dk, c.dv, c.ds):
        x.fill_(float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def call():
        snn.snn_linattn_fwd(c.d, c.q, c.k, c.v, c.decay, None, c.s0, c.o, c.s, c.ws)
        snn.snn_linattn_bwd(c.d, c.q, c.k, c.v, c.decay, None, c.s0, c.go, c.gs, c.dq, c.dk,
                            c.dv, c.ds, c.ws)

    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, (c.o, c.s, c.dq, c.dk, c.dv, c.ds)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        for x in (c.o, c.s, c.dq, c.dk, c.dv, c.ds):
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (c.o, c.s, c.dq, c.dk, c.dv, c.ds)):
            assert torch.equal(a, b)
