"""Linear attention of tokens and columns whose sizes differ by many powers of
two, within the bounds of ``test_gpu_linattn``: what a score, the state or a
value loses as a 16-bit operand is relative to its own token or column, not to
others'."""
import numpy as np
import pytest

from tests import block_reference as ref
from tests.test_gpu_linattn import TYPES, Case, _np

torch = pytest.importorskip("torch")
import paper_2211_10725_amd as snn  # noqa: E402

pytestmark = pytest.mark.gpu


def _rescaled(c, scale):
    c.scale = scale
    c.d = snn.linattn_desc(c.q, c.k, c.v, c.o, scale)
    return c


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("at", [5, 31, 75, 100])
@pytest.mark.parametrize("d", [64, 128])
def test_large_later_token_leaves_earlier_outputs(d, at, dt):
    """q = k = 6e4 of one token: the outputs before it stay as they are, bit for
    bit, and within their bounds."""
    c = Case(150, 1, 1, 1, d, d, dt, decay=[1.0])
    before = c.fwd()[0].clone()
    wo, _ = ref.linattn(*c.arrays())
    ao, _ = ref.linattn(*c.arrays(np.abs))
    c.q[at], c.k[at] = 6e4, 6e4
    o, _ = c.fwd()
    assert torch.equal(o[:at], before[:at])
    c.tol(_np(o[:at]), wo[:at], ao[:at])


@pytest.mark.parametrize("dt", list(TYPES))
def test_large_token_within_a_small_scale(dt):
    """The same with a scale that keeps every output in fp16's range: all tokens."""
    c = _rescaled(Case(150, 1, 1, 1, 64, 64, dt, decay=[0.9]), 2.0 ** -24)
    c.q[40], c.k[40] = 6e4, 6e4
    c.q[100, ..., 7] = -6e4
    c.check_fwd()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("at", [33, 40, 60])
def test_large_token_after_an_infinite_value(at, dt):
    """A chunk whose tokens go one by one for an infinity in v: a later token's
    size does not reach them either."""
    c = _rescaled(Case(150, 1, 1, 1, 64, 64, dt, decay=[1.0], state=False), 2.0 ** 10)
    c.q *= 2.0 ** -20
    wo, _ = ref.linattn(*c.arrays())
    ao, _ = ref.linattn(*c.arrays(np.abs))
    c.v[at - 1, 0, 0, 9] = float("inf")
    c.q[at], c.k[at] = 6e4, 6e4
    keep = [i for i in range(64) if i != 9]
    o, _ = c.fwd()
    c.tol(_np(o[:at - 1]), wo[:at - 1], ao[:at - 1])
    c.tol(_np(o[:at])[..., keep], wo[:at][..., keep], ao[:at][..., keep])


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,d", [(70, 64), (150, 128), (700, 64)])
def test_large_column_of_the_state_beside_ordinary_ones(T, d, dt):
    """The first state of 2^30 and -2^28 in one value of columns 3 and 8, which no
    query reads: the other columns' outputs keep their digits.  Within the two
    columns, two fp16 parts end at 2^-39 of the large value."""
    c = Case(T, 1, 2, 1, d, d, dt, decay=[1.0, 0.999])
    c.s0[:, :, 0, 3] = 2.0 ** 30
    c.s0[:, :, 0, 8] = -2.0 ** 28
    c.q[..., 0] = 0
    o, s = c.fwd()
    wo, ws = ref.linattn(*c.arrays())
    ao, as_ = ref.linattn(*c.arrays(np.abs))
    keep = [i for i in range(d) if i not in (3, 8)]
    c.tol(_np(o)[..., keep], wo[..., keep], ao[..., keep])
    c.tol(_np(s), ws, as_, fp32=True)
    if dt == "f16":  # in the bound as 2^-16 of its terms
        q = c.scale * np.abs(_np(c.q)).sum(3)
        ao[..., 3] += 2.0 ** (16 - 39 + 30) * q
        ao[..., 8] += 2.0 ** (16 - 39 + 28) * q
    c.tol(_np(o), wo, ao)


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,d", [(70, 64), (150, 128), (700, 64)])
def test_large_value_within_a_column(T, d, dt):
    """Two fp16 parts end at 2^-39 of the largest value of their own column, all
    that a small one may lose beside it: dq reads the state transposed, so its
    columns hold the 2^30 of the first state beside ordinary values."""
    c = Case(T, 1, 2, 1, d, d, dt, decay=[1.0, 0.999])
    c.s0[:, :, 0, 3] = 2.0 ** 30
    c.go[..., 3] = 0
    dq = _np(c.bwd()[0])
    z = np.zeros_like(_np(c.gs))
    want = ref.linattn_grads(*c.arrays(), _np(c.go), z)[0]
    absolute = ref.linattn_grads(*c.arrays(np.abs), np.abs(_np(c.go)), z)[0]
    rel, least = ref.HALF_ULP[dt]
    bound = ((2 * T + d + 24) * ref.EPS32 + 2.0 ** -16) * absolute + rel * np.abs(want) + least
    if dt == "f16":
        bound[..., 0] += 2.0 ** -39 * 2.0 ** 30 * c.scale * np.abs(_np(c.go)).sum(3)
    assert (np.abs(dq - want) <= bound).all()


def _columns(x, sizes):
    """The last dimension's values times powers of two in turn, as the type holds them."""
    f = torch.as_tensor(np.resize(sizes, x.shape[-1]), dtype=torch.float32, device=x.device)
    x.copy_((x.float() * f).to(x.dtype))


# fp16 holds 2^-24 to 65504; each size is beside every other within 16 columns
SIZES = [1.0, 2.0 ** 13, 2.0 ** -10, 2.0 ** -22, 1.0, 2.0 ** -16, 2.0 ** 10]


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("decay", [[1.0], [0.97]])
@pytest.mark.parametrize("T,d", [(70, 64), (150, 128), (700, 64)])
@pytest.mark.parametrize("what", ["v", "k", "q", "go"])
def test_columns_of_unequal_size(what, T, d, decay, dt):
    """Values, keys, queries or output gradients whose columns lie up to 2^35
    apart, over several chunks and segments: states and gradients of the small
    columns keep their digits."""
    c = _rescaled(Case(T, 1, 2, 1, d, d, dt, decay=decay), 2.0 ** -12)
    c.gs *= 2.0 ** -6  # gradients of at most 2^13 times it stay in fp16's range
    _columns(getattr(c, what), SIZES)
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("dt", list(TYPES))
def test_column_of_the_smallest_values_beside_the_largest(dt):
    """+-6e4 beside 2^-24 in neighbouring columns at decay 1: what every chunk adds
    to the small one stays in the state."""
    c = _rescaled(Case(200, 1, 1, 1, 64, 64, dt, decay=[1.0], state=False), 2.0 ** -6)
    sign = torch.as_tensor((-1.0) ** np.arange(200), device="cuda").view(200, 1, 1)
    c.v[..., 4] = (6e4 * sign).to(c.v.dtype)
    c.v[..., 5] = 2.0 ** -24
    c.k[:] = 1
    c.check_fwd()
    assert torch.equal(c.s[0, 0, :, 5], torch.full((64,), 200 * 2.0 ** -24, device="cuda"))
