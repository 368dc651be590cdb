"""Gates far from zero: 1 - s(z) of an open gate is known to as many places as s(z) of a closed one.

Tolerances, element by element and relative: exp(-z) is off by the rounding of its argument, |z| 2^-24, and one unit of the hardware's
exponential, the reciprocal by another, and a step has a handful of roundings: (16 + 2 |z|) 2^-24 for a step's factor, that many times for
a product of factors; and the rounding to the result's type (f16: 2^-25 absolutely among subnormal numbers)."""
import numpy as np
import pytest

import sequence_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LOW = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
TINY = {"bf16": 0.0, "f16": 2.0 ** -24, "f32": 2.0 ** -126}
GATES = (0.0, 0.5, 2.0, 4.0, 8.0, 11.0, 14.0, 17.0, 20.0, 40.0)


@pytest.fixture(scope="module")
def rb():
    from paper_2510_23498_amd import binding
    binding.load_library()
    return binding


def _np(t):
    return t.double().cpu().numpy()


def _near(got, want, low, steps, z, name):
    got, want = _np(got), np.asarray(want)
    off = np.abs(got - want)
    bound = (ref.UNIT[low] + steps * (16 + 2 * np.abs(z)) * 2.0 ** -24) * np.abs(want) + TINY[low]
    assert (off <= bound).all(), f"{name}: {(off / np.maximum(np.abs(want), 1e-300)).max():.3e} off"


def _channels(B, T, D, share, z):
    """Gates z, -z of channels in turn"""
    gates = torch.tensor([z, -z] * (D // share))[:D // share]
    return gates.expand(B, T, D // share).contiguous(), np.repeat(gates.numpy().astype(np.float64), share)


@pytest.mark.parametrize("z", GATES)
@pytest.mark.parametrize("low", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("share", [1, 2, 16])
def test_gradients_of_one_step(rb, low, z, share):
    B, D = 3, 64
    rng = np.random.default_rng(int(8 * z) + share)
    g = lambda *s: torch.from_numpy(rng.uniform(0.5, 1.5, s).astype(np.float32))  # noqa: E731
    zt, zn = _channels(B, 1, D, share, z)
    x, dh = g(B, 1, D).to(LOW[low]).cuda(), g(B, 1, D).to(LOW[low]).cuda()
    h0, dhT, zt = -g(B, D).cuda(), g(B, D).cuda(), zt.to(LOW[low]).cuda()   # (all terms of one sign: nothing cancels)
    h, hT, states = rb.rampde_recurrence_fwd(x, zt, h0=h0, save_states=True)
    dx, dz, dh0 = rb.rampde_recurrence_bwd(x, zt, states, dh, dhT=dhT, h0=h0)
    wh, wT, wdx, wdz, wdh0 = ref.recurrence(_np(x), _np(zt), _np(h0), None, _np(dh), _np(dhT))
    if share == 1:   # (1 - s subtracts in the reference too, which 64 bits leave room for up to z = 20)
        s, c = 1 / (1 + np.exp(-zn)), 1 / (1 + np.exp(zn))
        G = _np(dh)[:, 0] + _np(dhT)
        wdz, wdh0 = (G * (_np(x)[:, 0] - _np(h0)) * s * c)[:, None], G * c
    _near(dx, wdx, low, 1, z, "dx")
    if share == 1 or z <= 20:
        _near(dz, wdz, low, 1, z, "dz")
        _near(dh0, wdh0, "f32", 1, z, "dh0")


@pytest.mark.parametrize("z", [2.0, 4.0, 8.0])
@pytest.mark.parametrize("D", [128, 63])
def test_what_open_gates_leave_of_the_last_gradient(rb, z, D):
    """No gradient but the last one's: products of 1 - s over the steps, fp32 (inputs of alternating signs, so that x - h is large)"""
    T = 9
    x = (torch.tensor([1.5, -1.5] * 5)[:T, None] * torch.ones(2, T, D)).cuda()
    zt, h0 = torch.full((2, T, D), z, device="cuda"), torch.full((2, D), -1.0, device="cuda")
    dhT = torch.full((2, D), 3.0, device="cuda")
    states = rb.rampde_recurrence_fwd(x, zt, h0=h0, save_states=True)[2]
    dx, dz, dh0 = rb.rampde_recurrence_bwd(x, zt, states, None, dhT=dhT, h0=h0)
    c, s = 1 / (1 + np.exp(z)), 1 / (1 + np.exp(-z))
    G = 3 * c ** np.arange(T - 1, -1, -1)[None, :, None] * np.ones((2, T, D))
    h = ref.recurrence(_np(x), _np(zt), _np(h0))[0]
    before = np.concatenate([_np(h0)[:, None], h[:, :-1]], 1)
    _near(dx, G * s, "f32", T, z, "dx")
    _near(dh0, 3 * c ** T * np.ones((2, D)), "f32", T, z, "dh0")
    _near(dz, G * (_np(x) - before) * s * c, "f32", T + 2, z, "dz")


@pytest.mark.parametrize("T", [40, 300, 2500])
@pytest.mark.parametrize("low", ["bf16", "f16", "f32"])
def test_gradients_of_open_gates_along_a_sequence(rb, low, T):
    """Inputs of alternating signs (so that x - h does not cancel) and gradients of one sign, gates of 6 to 16, several tiles"""
    B, D = 2, 130
    rng = np.random.default_rng(T)
    sign = torch.tensor([1.0, -1.0] * ((T + 1) // 2))[:T, None]
    x = (torch.from_numpy(rng.uniform(1, 2, (B, T, D)).astype(np.float32)) * sign).to(LOW[low]).cuda()
    z = torch.from_numpy(rng.uniform(6, 16, (B, T, D)).astype(np.float32)).to(LOW[low]).cuda()
    dh = torch.from_numpy(rng.uniform(0.5, 1.5, (B, T, D)).astype(np.float32)).to(LOW[low]).cuda()
    h0 = torch.full((B, D), -1.0, device="cuda")
    h, hT, states = rb.rampde_recurrence_fwd(x, z, h0=h0, save_states=True)
    dx, dz, dh0 = rb.rampde_recurrence_bwd(x, z, states, dh, h0=h0)
    zn, xn = _np(z), _np(x)
    want = ref.recurrence(xn, zn, _np(h0), None, _np(dh))
    # (the reference's 1 - s is off by 2^-53 exp(16), 1e-9, relatively)
    _near(h, want[0], low, 2, zn, "h")
    _near(dx, want[2], low, 2, zn, "dx")
    _near(dz, want[3], low, 4, zn, "dz")
    _near(dh0, want[4], "f32", 2, 16.0, "dh0")


@pytest.mark.parametrize("rows,cols", [(6, 40), (5, 200), (4, 512), (3, 1001), (2, 8192), (2, 9000)])
@pytest.mark.parametrize("low", ["bf16", "f16", "f32"])
def test_gate_gradients_of_a_join(rb, low, rows, cols):
    """Branch, parameters and gradient of y' of one sign, no gradient of x: nothing cancels in dgate.  The gates of a row go over the whole
    range, both signs."""
    rng = np.random.default_rng(cols)
    g = lambda *s: torch.from_numpy(rng.uniform(0.5, 1.5, s).astype(np.float32)).cuda()  # noqa: E731
    z = np.resize(np.concatenate([GATES, [-v for v in GATES]]), (rows, cols))
    y, b, gate, dy = g(rows, cols), g(rows, cols).to(LOW[low]), torch.from_numpy(z.astype(np.float32)).to(LOW[low]).cuda(), g(rows, cols)
    w_post, scale = g(cols), g(cols)
    j = rb.Join(alpha=0.5, eps=1e-5)
    y2, _, rstd = rb.rampde_join_fwd(j, y, b, gate=gate, w_post=w_post, scale=scale, want_x=False, save_rstd=True)
    got = rb.rampde_join_bwd(j, y2, b, rstd, dy, None, gate=gate, w_post=w_post, scale=scale).dgate
    n = _np(b) / np.sqrt((_np(b) ** 2).mean(1, keepdims=True) + 1e-5)
    want = 0.5 * _np(dy) * _np(scale) * n * _np(w_post) / (1 + np.exp(-z)) / (1 + np.exp(z))
    # (the row's norm: a sum of squares in fp32, sqrt(cols) 2^-24)
    _near(got, want, low, 1 + np.sqrt(cols) / 16, z, "dgate")


def test_gate_gradients_of_closed_and_missing_gates(rb):
    """Past the range of exp: s is 0, its derivative too, and a NaN shows"""
    y, b, dy = torch.ones(1, 8, device="cuda"), torch.ones(1, 8, device="cuda"), torch.ones(1, 8, device="cuda")
    gate = torch.tensor([[-87.0, -87.7, -88.5, -100.0, float("-inf"), 100.0, float("inf"), float("nan")]], device="cuda")
    y2, _, rstd = rb.rampde_join_fwd(rb.Join(), y, b, gate=gate, want_x=False, save_rstd=True)
    got = rb.rampde_join_bwd(rb.Join(), y2, b, rstd, dy, None, gate=gate).dgate[0]
    assert (got[:7].abs() <= 2e-38).all() and torch.isnan(got[7])


def test_gates_of_fp32_operands_over_their_whole_range(rb):
    """Relative error that does not grow with |z|: one unit each of exponential and reciprocal (2^-23) and a handful of roundings, 8 of
    2^-24 for s, 20 for products of s, 1 - s and two more factors.  (The reference forms s and 1 - s without subtractions.)"""
    z = np.concatenate([np.linspace(-80, 80, 1281), np.linspace(-1, 1, 255)]).astype(np.float32).astype(np.float64)
    s, c, D = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z)), len(z)
    zt, one = torch.from_numpy(z.astype(np.float32)).cuda(), torch.ones(1, 1, D, device="cuda")
    h, hT, states = rb.rampde_recurrence_fwd(one, zt.view(1, 1, D), save_states=True)
    dx, dz, dh0 = rb.rampde_recurrence_bwd(one, zt.view(1, 1, D), states, one, h0=torch.zeros(1, D, device="cuda"))
    y, b = torch.zeros(1, D, device="cuda"), torch.ones(1, D, device="cuda")
    y2, _, rstd = rb.rampde_join_fwd(rb.Join(eps=1e-30), y, b, gate=zt.view(1, D), want_x=False, save_rstd=True)
    dgate = rb.rampde_join_bwd(rb.Join(eps=1e-30), y2, b, rstd, b, None, gate=zt.view(1, D)).dgate
    for got, want, n in ((h, s, 8), (hT, s, 8), (dx, s, 8), (dh0, c, 8), (dz, s * c, 20), (y2, s, 12), (dgate, s * c, 20)):
        assert np.max(np.abs(_np(got).ravel() / want - 1)) <= n * 2.0 ** -24
